// Scores of cached tokens and the choice among them (fw_cache_scores,
// fw_cache_select).
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// scores
//
//   s_j = 1/R sum_r [r sees j] exp(scale_h 2^ek(j) <q_r, code_j> - lse_r)
//
// over a cell's R rows (T positions x G heads).  A wave takes 64 tokens: their
// codes become bf16 (exact) once, in registers, and meet the rows tile by tile
// from LDS, S = Q K^T on 16x16x32 MFMA: a lane's four results are four rows of
// one token, so the sum over rows stays in the lane.  lse is known, so nothing
// is kept but the sums.  Float32 queries are taken apart into three bf16
// parts, which hold all 24 bits.  More rows than the workgroup's LDS holds are
// taken in turns, which add to what the turn before wrote.
// ---------------------------------------------------------------------------
constexpr int SW = 4;          // waves of a workgroup
constexpr int ST = 64 * SW;
constexpr int TT = 64;         // tokens of a wave and step
constexpr int kQBytes = 65536; // rows in LDS at a time
constexpr int kShares = 512;   // workgroups that share the tokens
constexpr int kLeast = 4;      // tiles of a workgroup at least
constexpr float SLOG2E = 1.4426950408889634f;

struct ScoreArgs {
    const void *q;
    int64_t q_seq, q_tok, q_head;
    int C, T, Hkv, G, W, R, d, turn;   // turn: rows in LDS at a time, a multiple of 16
    const uint8_t *kc, *k_exp;
    int64_t n_blocks;
    int shift;
    const int32_t *table, *lens;
    const float *scale, *lse, *earlier;
    float *scores;
    int64_t n;
};

__device__ __forceinline__ int scored(const ScoreArgs &a, int c) {  // tokens of a cell that are scored
    const int64_t most = (int64_t)a.W << a.shift, cap = most < a.n ? most : a.n;
    const int len = a.lens[c];
    return len < 0 ? 0 : len > cap ? (int)cap : len;
}
__device__ __forceinline__ int cell_len(const ScoreArgs &a, int c) {
    const int64_t most = (int64_t)a.W << a.shift;
    const int len = a.lens[c];
    return len < 0 ? 0 : len > most ? (int)most : len;
}
__device__ __forceinline__ float exp2_of_byte(int b) { return __uint_as_float((uint32_t)(b < 1 ? 1 : b) << 23); }

__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], e[0], e[1]};
}

template <typename T, int DP>
__global__ void __launch_bounds__(ST) cache_scores(ScoreArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;            // bf16 parts of a query
    constexpr int KS = DP / 32, KB = DP / 4, KW = KB / 4;  // key steps; bytes and words of a lane's part of a key
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ int red[ST / 64], found[2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tl = lane & 15, g = lane >> 4;
    bf16x8 *const qs = (bf16x8 *)lds;                          // [row tile][key step][part][lane]
    float *const ls = (float *)(lds + (size_t)a.turn * KS * NP * 64);  // [row] lse, base 2
    int *const back = (int *)(ls + a.turn);                    // [row] last tokens that it does not see

    // this workgroup's tiles of all cells' in a row
    const int run = (a.C + ST - 1) / ST, c0 = tid * run, c1 = c0 + run < a.C ? c0 + run : a.C;
    int mine = 0;
    for (int c = c0; c < c1; ++c) mine += (scored(a, c) + TT - 1) / TT;
    int x = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    if (lane == 63) red[w] = x;
    __syncthreads();
    int first = x - mine, all = 0;
#pragma unroll
    for (int i = 0; i < SW; ++i) {
        if (i < w) first += red[i];
        all += red[i];
    }
    const int per = max((all + (int)gridDim.x - 1) / (int)gridDim.x, kLeast);
    if ((int64_t)blockIdx.x * per >= all) return;
    const int g0 = blockIdx.x * per, g1 = min(g0 + per, all);
    if (g0 >= first && g0 < first + mine)
        for (int c = c0; c < c1; ++c) {
            const int n = (scored(a, c) + TT - 1) / TT;
            if (g0 < first + n) {
                found[0] = c, found[1] = first;
                break;
            }
            first += n;
        }
    __syncthreads();
    int c = __builtin_amdgcn_readfirstlane(found[0]), at = __builtin_amdgcn_readfirstlane(found[1]);
    const float mean = 1.f / a.R;
    const int bmask = (1 << a.shift) - 1;

    for (; c < a.C && at < g1; ++c) {
        const int n = scored(a, c), nt = (n + TT - 1) / TT;
        const int t0 = max(g0 - at, 0), t1 = min(g1 - at, nt);
        at += nt;
        if (t0 >= t1) continue;
        const int len = cell_len(a, c), seq = c / a.Hkv, h = c % a.Hkv;
        const int32_t *row = a.table + (int64_t)c * a.W;
        const float sl2 = (a.scale ? a.scale[h] : (float)(1.0 / sqrt((double)a.d))) * SLOG2E;
        for (int r0 = 0; r0 < a.R; r0 += a.turn) {
            const int rows = min(a.turn, a.R - r0), tiles = (rows + 15) / 16;
            __syncthreads();  // the rows before are done with
            for (int i = tid; i < tiles * KS * 64; i += ST) {
                const int l = i & 63, y = (i >> 6) % KS, rt = (i >> 6) / KS;
                const int r = r0 + 16 * rt + (l & 15), col = KB * (l >> 4) + 8 * y;
                const T *p = (const T *)a.q + seq * a.q_seq + (r / a.G) * a.q_tok + (h * a.G + r % a.G) * a.q_head;
                bf16x8 z[NP];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float v = r < a.R && col + k < a.d ? Elem<T>::load(p, col + k) : 0.f;
#pragma unroll
                    for (int s = 0; s < NP; ++s) {
                        z[s][k] = (__bf16)v;
                        v -= (float)z[s][k];
                    }
                }
#pragma unroll
                for (int s = 0; s < NP; ++s) qs[((rt * KS + y) * NP + s) * 64 + l] = z[s];
            }
            for (int i = tid; i < 16 * tiles; i += ST) {
                const int r = r0 + i;
                const bool in = r < a.R;
                ls[i] = in ? a.lse[((int64_t)seq * a.T + r / a.G) * a.Hkv * a.G + h * a.G + r % a.G] * SLOG2E : INFINITY;
                back[i] = in ? a.T - 1 - r / a.G : len;
            }
            __syncthreads();
            const int full = len - (a.T - 1);  // tokens that every row sees
            for (int t = t0 + w; t < t1; t += SW) {
                const int base = t * TT;
                bf16x8 kf[4][KS];
                float f[4];
                bool in[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int tok = base + 16 * x + tl, b = tok < len ? row[tok >> a.shift] : -1;
                    in[x] = b >= 0 && b < a.n_blocks;
                    const int64_t bb = in[x] ? b : 0;
                    const uint8_t *p = a.kc + ((bb << a.shift) + (tok & bmask)) * DP + KB * g;
                    f[x] = sl2 * exp2_of_byte(a.k_exp[bb]);
                    uint32_t kr[KW];
#pragma unroll
                    for (int y = 0; y < KW; y += (KW % 4 == 0 ? 4 : 2)) {
                        if constexpr (KW % 4 == 0) *(uint4 *)&kr[y] = *(const uint4 *)(p + 4 * y);
                        else *(uint2 *)&kr[y] = *(const uint2 *)(p + 4 * y);
                    }
#pragma unroll
                    for (int y = 0; y < KS; ++y) kf[x][y] = widen(kr[2 * y], kr[2 * y + 1]);
                }
                const bool masked = base + TT > full;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
                for (int rt = 0; rt < tiles; ++rt) {
                    f32x4 s[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) s[x] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int y = 0; y < KS; ++y)
#pragma unroll
                        for (int z = NP - 1; z >= 0; --z) {
                            const bf16x8 qf = qs[((rt * KS + y) * NP + z) * 64 + lane];
#pragma unroll
                            for (int x = 0; x < 4; ++x) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf, kf[x][y], s[x], 0, 0, 0);
                        }
                    const f32x4 l = *(const f32x4 *)(ls + 16 * rt + 4 * g);
                    if (masked) {
                        const int4 bk = *(const int4 *)(back + 16 * rt + 4 * g);
                        const int hid[4] = {len - bk.x, len - bk.y, len - bk.z, len - bk.w};
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float e = __builtin_amdgcn_exp2f(fmaf(s[x][i], f[x], -l[i]));
                                sum[x] += base + 16 * x + tl < hid[i] ? e : 0.f;
                            }
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[x] += __builtin_amdgcn_exp2f(fmaf(s[x][i], f[x], -l[i]));
                    }
                }
                float out = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float y = in[x] ? sum[x] : 0.f;
                    y += __shfl_xor(y, 16);
                    y += __shfl_xor(y, 32);
                    out = g == x ? y : out;
                }
                const int tok = base + lane;  // 16 g + tl
                if (tok < n) {
                    const int64_t i = c * a.n + tok;
                    const float old = r0 > 0 ? a.scores[i] : a.earlier ? a.earlier[i] : 0.f;
                    a.scores[i] = fmaf(out, mean, old);
                }
            }
        }
    }
}

template <typename T, int DP>
hipError_t launch_scores_width(ScoreArgs &a, hipStream_t st) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;
    const int row = 2 * DP * NP;
    a.turn = std::min((a.R + 15) / 16 * 16, kQBytes / row / 16 * 16);
    const size_t lds = (size_t)a.turn * (row + 8);
    const int64_t tiles = (int64_t)a.C * ((std::min<int64_t>((int64_t)a.W << a.shift, a.n) + TT - 1) / TT);
    const unsigned grid = (unsigned)std::min<int64_t>(kShares, (tiles + kLeast - 1) / kLeast);
    hipLaunchKernelGGL((cache_scores<T, DP>), dim3(grid), dim3(ST), lds, st, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// select
//
// The last `recent` kept tokens are certain; of those before them the rest of
// keep[c] is chosen by the key of the score, found 11, 11 and 10 bits at a time
// from a histogram, and then, among equal keys, by position.
// ---------------------------------------------------------------------------
constexpr int LT = 1024;  // threads of a workgroup
constexpr int kBins = 2048;

struct SelectArgs {
    int64_t C, n, n_kept;
    const float *scores;
    const int32_t *lens, *keep;
    int64_t recent;
    int64_t *offsets;
    int32_t *kept_pos;
};

__device__ __forceinline__ uint32_t rank_key(float x) { return x != x ? 0xFFFFFFFFu : ord_key(x); }
__device__ __forceinline__ int kept_of(const SelectArgs &a, int64_t c, int *len) {
    const int64_t l = a.lens[c];
    const int n = l < 0 ? 0 : l > a.n ? (int)a.n : (int)l, k = a.keep[c];
    *len = n;
    return k < 0 ? 0 : k > n ? n : k;
}

template <int NT, typename V>
__device__ __forceinline__ V scan_before(V v, V *red, V *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    V x = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const V y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    if (lane == 63) red[w] = x;
    __syncthreads();
    V before = x - v, all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        const V y = red[i];
        if (i < w) before += y;
        all += y;
    }
    __syncthreads();
    *total = all;
    return before;
}

__global__ void __launch_bounds__(LT) select_offsets(SelectArgs a) {
    __shared__ int64_t red[LT / 64];
    const int64_t run = (a.C + LT - 1) / LT, c0 = threadIdx.x * run, c1 = c0 + run < a.C ? c0 + run : a.C;
    int64_t mine = 0, all;
    int len;
    for (int64_t c = c0; c < c1; ++c) mine += kept_of(a, c, &len);
    int64_t at = scan_before<LT, int64_t>(mine, red, &all);
    for (int64_t c = c0; c < c1; ++c) {
        a.offsets[c] = at;
        at += kept_of(a, c, &len);
    }
    if (threadIdx.x == 0) a.offsets[a.C] = all;
}

__global__ void __launch_bounds__(LT) cache_select(SelectArgs a) {
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t red[LT / 64];
    __shared__ uint32_t s_bin, s_above;
    const int tid = threadIdx.x;
    const int64_t c = blockIdx.x;
    // behind the last kept token
    for (int64_t i = a.offsets[a.C] + c * LT + tid; i < a.n_kept; i += (int64_t)gridDim.x * LT) a.kept_pos[i] = -1;
    int len;
    const int keep = kept_of(a, c, &len);
    const int certain = (int)(a.recent < keep ? a.recent : keep), nf = len - certain, need = keep - certain;
    const int64_t o = a.offsets[c];
    for (int i = tid; i < certain; i += LT)
        if (o + need + i < a.n_kept) a.kept_pos[o + need + i] = nf + i;
    if (need == 0) return;
    const float *row = a.scores + c * a.n;
    uint32_t key = 0, mask = 0, rem = need;
    if (need < nf) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t dm = pass == 2 ? 1023u : 2047u;
            for (int i = tid; i < kBins; i += LT) hist[i] = 0;
            __syncthreads();
            for (int j = tid; j < nf; j += LT) {
                const uint32_t u = rank_key(row[j]);
                if ((u & mask) == key) atomicAdd(&hist[(u >> shift) & dm], 1u);
            }
            __syncthreads();
            // two bins a thread, from the top
            const uint32_t h0 = hist[kBins - 1 - 2 * tid], h1 = hist[kBins - 2 - 2 * tid];
            uint32_t all;
            const uint32_t before = scan_before<LT, uint32_t>(h0 + h1, red, &all);
            if (before < rem && rem <= before + h0) s_bin = kBins - 1 - 2 * tid, s_above = before;
            else if (before + h0 < rem && rem <= before + h0 + h1) s_bin = kBins - 2 - 2 * tid, s_above = before + h0;
            __syncthreads();
            key |= s_bin << shift, mask |= dm << shift, rem -= s_above;
        }
    }
    // those above the key, and the first rem of those at it
    int64_t at = o;
    uint32_t seen = 0;
    for (int j0 = 0; j0 < nf; j0 += LT) {
        const int j = j0 + tid;
        const uint32_t u = j < nf ? rank_key(row[j]) : 0;
        const bool more = j < nf && (need == nf || u > key), same = j < nf && need < nf && u == key;
        uint32_t all;
        const uint32_t before = scan_before<LT, uint32_t>((uint32_t)more | (uint32_t)same << 16, red, &all);
        const uint32_t eq = seen + (before >> 16), taken = (before & 0xFFFFu) + (min(eq, rem) - min(seen, rem));
        if ((more || (same && eq < rem)) && at + taken < a.n_kept) a.kept_pos[at + taken] = j;
        const uint32_t upto = seen + (all >> 16);
        at += (all & 0xFFFFu) + (min(upto, rem) - min(seen, rem));
        seen = upto;
    }
}
}  // namespace

hipError_t launch_cache_scores(const fw_cache &cache, int dtype, const void *q, int64_t S, int64_t T, int64_t Hq,
                               int64_t Hkv, int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table,
                               int64_t W, const int32_t *lens, const float *scale, const float *lse,
                               const float *earlier, float *scores, int64_t n, hipStream_t st) {
    ScoreArgs a{};
    a.q = q, a.q_seq = q_seq, a.q_tok = q_tok, a.q_head = q_head;
    a.C = (int)(S * Hkv), a.T = (int)T, a.Hkv = (int)Hkv, a.G = (int)(Hq / Hkv), a.W = (int)W;
    a.R = a.T * a.G, a.d = (int)cache.d;
    a.kc = cache.k, a.k_exp = cache.k_exp, a.n_blocks = cache.n_blocks, a.shift = __builtin_ctz(cache.block_size);
    a.table = table, a.lens = lens, a.scale = scale, a.lse = lse, a.earlier = earlier, a.scores = scores, a.n = n;
    const auto width = [&](auto t) {
        using E = decltype(t);
        switch (cache_row(cache.d)) {
            case 32: return launch_scores_width<E, 32>(a, st);
            case 64: return launch_scores_width<E, 64>(a, st);
            case 96: return launch_scores_width<E, 96>(a, st);
            case 128: return launch_scores_width<E, 128>(a, st);
            case 192: return launch_scores_width<E, 192>(a, st);
            default: return launch_scores_width<E, 256>(a, st);
        }
    };
    return dtype == FW_F32 ? width(float()) : width(uint16_t());
}

hipError_t launch_select_cells(int64_t C, const float *scores, int64_t n, const int32_t *lens, const int32_t *keep,
                               int64_t recent, int64_t n_kept, int64_t *offsets, int32_t *kept_pos, hipStream_t st) {
    SelectArgs a{C, n, n_kept, scores, lens, keep, recent, offsets, kept_pos};
    hipLaunchKernelGGL(select_offsets, dim3(1), dim3(LT), 0, st, a);
    hipLaunchKernelGGL(cache_select, dim3((unsigned)C), dim3(LT), 0, st, a);
    return hipGetLastError();
}

}  // namespace fw
