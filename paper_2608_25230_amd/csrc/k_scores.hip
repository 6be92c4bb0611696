// Scores of cached tokens and the choice among them (fw_cache_scores,
// fw_cache_select).
#include <algorithm>
#include <type_traits>

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
// codes become bf16 (exact) in registers and meet the rows 16 at a time, S = Q
// K^T on 16x16x32 MFMA: a lane's four results are four rows of one token, so
// the sum over rows stays in the lane.  lse is known, so nothing is kept but
// the sums.  Float32 queries are taken apart into three bf16 parts, which hold
// all 24 bits.
//
// Cells differ in length, so the work is cut by length, on the device: all
// cells' tiles of 64 tokens in a row, the same number to each workgroup.  A
// cell's first share costs more than its tiles, which many_rows counts in
// (kFill).  Its time goes by rounds of a tile for each wave, not by tiles, which
// cells of a few thousand tokens feel: 64 of 4000, 128 rows, are shares of 9 tiles
// for 8 waves (26 us; its products alone 6).
//
// few_rows, up to 16 rows a cell: a wave holds them in registers; keys are loaded
// a tile ahead.  Memory bounds it: 512 cells of 3000 to 30000 tokens of 128
// columns, 4 rows, 438 MB in 95.5 us (4.6 TB/s; 5.8 once it runs, after 15 us in
// which shares are found and the first keys come).  The older waves of a compute
// unit are served first, so a workgroup takes all of it and its waves take tiles
// one by one: with a fixed share each the first were done at two thirds of the
// time (98 us; 16384 cells of 200 tokens 113 instead of 64).  By many_rows 128
// cells of 8000 tokens and 1 to 16 rows take 32 us instead of 25 to 28.
//
// many_rows: a workgroup's waves share the rows in LDS; more rows than it holds
// are taken in turns, which add to what the turn before wrote.  Matrix and vector
// units bound it together, which run side by side only in part: 64 tokens x 16
// rows of 128 columns take 16 matrix instructions and as many products with the
// scale, exponentials and sums, in a bare loop on registers about 200 ns a SIMD,
// here 228 (256 cells of 3000 to 30000 tokens, 256 rows: 102 GFLOP of products in
// 120 us).  Slower were: the next tile's keys loaded ahead by waves of twice the
// registers (132), a tile's products between the weights of the one before (125
// to 133), keys staged in LDS for all waves instead of rows (150 to 170).
// ---------------------------------------------------------------------------
constexpr int TT = 64;          // tokens of a wave and step
// its workgroups: one to a compute unit, whose registers its waves fill; twice as many take 98 us at the size above, and
// 128 cells of 8000 tokens 33 us instead of 27
constexpr int kFewGroups = 256;
// many_rows: rows in LDS at a time, so that two workgroups fit a compute unit and one loads rows while the other computes.
// Where they do not hold all rows, one workgroup of twice the waves holds twice as many and takes fewer turns (64 cells of
// 4000 tokens, 512 / 2048 rows: 60 / 207 us, by two 64 / 220; float32, 128 rows: 36 and 40; 256 columns, 512 rows: 94 and
// 108).  Where they do, two are better (2048 cells of 500 tokens, 20 rows: 48 us, by one 61).
constexpr int kQBytes = 65536;
// two to a compute unit: 138 us at the size above on one card; three in turns 152, four 160
constexpr int kManyGroups = 512;
// tiles of a workgroup at least (8 cells of 4000 tokens, 256 rows: 16 us; one 19.5, four 17.7, eight 22)
constexpr int kManyLeast = 2;
// what a cell's rows cost there, in tiles: 8 127 to 134 us at the size above; 0 136 to 151, 4 139 to 143, 16 134 to 143
constexpr int kFill = 8;
constexpr float SLOG2E = 1.4426950408889634f;

struct ScoreArgs {
    const void *q;
    int64_t q_seq, q_tok, q_head;
    int C, T, Hkv, G, W, R, d, turn;  // turn: rows in LDS at a time, a multiple of 16
    const uint8_t *kc, *k_exp;
    int64_t n_blocks;
    int shift;
    const int32_t *table, *lens;
    const float *scale, *lse, *earlier;
    float *scores;
    int64_t n;
    bool wide;  // 16-byte aligned queries of a multiple of 8 columns
};

__device__ __forceinline__ int cell_len(const ScoreArgs &a, int c) {
    const int64_t most = (int64_t)a.W << a.shift;
    const int len = a.lens[c];
    return len < 0 ? 0 : len > most ? (int)most : len;
}
__device__ __forceinline__ int scored(const ScoreArgs &a, int c) {  // tokens of a cell that are scored
    const int len = cell_len(a, c);
    return len > a.n ? (int)a.n : len;
}
// Tiles of n tokens.  A cell may hold 2^31 - 1 of them: counts that round up are unsigned, and no token number goes past
// the last tile's.
__device__ __forceinline__ int tile_count(int n) { return (int)(((uint32_t)n + TT - 1) / TT); }
__device__ __forceinline__ float exp2_of_byte(int b) { return __uint_as_float((uint32_t)(b < 1 ? 1 : b) << 23); }

__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], e[0], e[1]};
}

// Shares [g0, g1) of the cells' tiles, EXTRA more for what a cell costs besides them, N to a workgroup, share i of
// workgroup b being number b N + i of `shares`: each share's first cell and the first tile of that.  found[i] = (cell, its
// first tile), cell -1 where the share is empty.
template <int NT, int N, int EXTRA>
__device__ __forceinline__ void find_shares(const ScoreArgs &a, int shares, int least, int2 (&found)[N], int *per) {
    __shared__ int red[NT / 64];
    __shared__ int2 got[N];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int run = (a.C + NT - 1) / NT, c0 = tid * run, c1 = c0 + run < a.C ? c0 + run : a.C;
    int mine = 0;
    const auto tiles_of = [&](int c) {
        const int n = tile_count(scored(a, c));
        return n > 0 ? n + EXTRA : 0;
    };
    for (int c = c0; c < c1; ++c) mine += tiles_of(c);
    int x = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    if (lane == 63) red[w] = x;
    if (tid < N) got[tid].x = -1;
    __syncthreads();
    int first = x - mine, all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        if (i < w) first += red[i];
        all += red[i];
    }
    *per = max((int)(((int64_t)all + shares - 1) / shares), least);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t g = ((int64_t)blockIdx.x * N + i) * *per;
        if (g < first || g >= first + mine) continue;
        int at = first;
        for (int c = c0; c < c1; ++c) {
            const int n = tiles_of(c);
            if (g < at + n) {
                got[i] = make_int2(c, at);
                break;
            }
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) found[i] = got[i];
}

// The 16 tokens of piece x of tile t lie in one block: its number, the same for the whole wave, or -1.
__device__ __forceinline__ int page_of(const ScoreArgs &a, const int32_t *row, int len, int t, int x) {
    const uint32_t tok = (uint32_t)t * TT + 16 * x;  // of a tile that a wave looks ahead to, maybe past 2^31
    const int b = tok < (uint32_t)len ? row[tok >> a.shift] : -1;
    return b >= 0 && b < a.n_blocks ? b : -1;
}

// A lane's part of a tile's keys: token 16 x + lane % 16, and a quarter of its columns, by loads of 16 bytes (8 where rows
// are no multiple of 64).  NEAR: a lane's bytes are neighbours, which many_rows does better with (64 cells of 4000 tokens,
// 2048 rows of 128 columns: 216 us, else 222); otherwise the lane groups' bytes of a load are (512 cells of 8000 tokens of
// 256 columns, 4 rows: 212 us, else 230; of 128 columns the same).
template <int DP, bool NEAR>
struct Keys {
    static constexpr int KW = DP / 16;                // words
    static constexpr int LW = KW % 4 == 0 ? 4 : 2;    // words of a load
    static constexpr int STEP = NEAR ? 4 : 16;        // bytes from a load to the next, for each of its words
    static constexpr int GROUP = NEAR ? DP / 4 : 4 * LW;  // and from a lane group to the next
    uint32_t k[4][KW];
    int e[4];
    // first column of key step y
    static __device__ __forceinline__ int column(int y, int g) { return STEP * (2 * y / LW * LW) + GROUP * g + 8 * y % (4 * LW); }
    __device__ __forceinline__ void load(const ScoreArgs &a, int t, const int (&page)[4], int lane) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int64_t b = page[x] < 0 ? 0 : page[x];
            const uint8_t *p = a.kc + ((b << a.shift) + ((t * TT + 16 * x) & ((1 << a.shift) - 1))) * DP + (lane & 15) * DP +
                               GROUP * (lane >> 4);
#pragma unroll
            for (int y = 0; y < KW; y += LW) {
                if constexpr (LW == 4) *(uint4 *)&k[x][y] = *(const uint4 *)(p + STEP * y);
                else *(uint2 *)&k[x][y] = *(const uint2 *)(p + STEP * y);
            }
            e[x] = a.k_exp[b];
        }
    }
};

// Eight columns of row r of a cell as bf16 parts; zeros past the rows and columns there are.
template <typename T, int NP>
__device__ __forceinline__ void load_row(const ScoreArgs &a, const T *p, bool in, int col, bf16x8 (&z)[NP]) {
    if (NP == 1 && a.wide) {
        uint4 v = {0u, 0u, 0u, 0u};
        if (in && col < a.d) v = *(const uint4 *)(p + col);
        z[0] = __builtin_bit_cast(bf16x8, v);
        return;
    }
    float v[8];
    if (a.wide) {
        f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
        if (in && col < a.d) lo = *(const f32x4 *)(p + col), hi = *(const f32x4 *)(p + col + 4);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < 4 ? lo[k & 3] : hi[k & 3];
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = in && col + k < a.d ? Elem<T>::load(p, col + k) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            z[s][k] = (__bf16)v[k];
            v[k] -= (float)z[s][k];
        }
}

// Adds e^(z - lse) of 16 rows to the lane's tokens' sums; hid: the first token that each of the lane's four rows does not see.
template <bool MASKED>
__device__ __forceinline__ void add_weights(const f32x4 (&s)[4], const f32x4 &l, const float (&f)[4], const int (&hid)[4], int tok,
                                            float (&sum)[4]) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[x][i], f[x], -l[i]));
            sum[x] += !MASKED || tok + 16 * x < hid[i] ? e : 0.f;
        }
}

// A tile's scores: the sums of the lane groups together, times 1 / R, and what was there before.
__device__ __forceinline__ void put_scores(const ScoreArgs &a, int64_t at, const float (&sum)[4], const int (&page)[4], int lane,
                                           bool in, float mean, float old) {
    float out = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        float y = page[x] >= 0 ? sum[x] : 0.f;
        y += __shfl_xor(y, 16);
        y += __shfl_xor(y, 32);
        out = (lane >> 4) == x ? y : out;
    }
    if (in) a.scores[at] = fmaf(out, mean, old);
}

// NW waves, which take their workgroup's tiles one by one.
struct Tile {
    int c, t, len;  // cell (-1: none), tile of it, its length
};
template <typename T, int DP, int NW>
__global__ void __launch_bounds__(64 * NW, NW / 4) few_rows(ScoreArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, KS = DP / 32;  // bf16 parts of a query, key steps
    __shared__ int taken;
    const int lane = threadIdx.x & 63, tl = lane & 15, g = lane >> 4;
    if (threadIdx.x == 0) taken = 0;
    int2 found[1];
    int per;
    find_shares<64 * NW, 1, 0>(a, gridDim.x, 1, found, &per);
    int c = __builtin_amdgcn_readfirstlane(found[0].x), at = __builtin_amdgcn_readfirstlane(found[0].y);
    if (c < 0) return;
    const int g0 = blockIdx.x * per;  // below 2^30 tiles
    const float mean = 1.f / a.R;
    int len = cell_len(a, c), nt = tile_count(scored(a, c));  // of cell c, whose first tile is number `at`
    const auto take = [&]() -> Tile {
        int k = 0;
        if (lane == 0) k = atomicAdd(&taken, 1);
        k = __builtin_amdgcn_readfirstlane(k);
        if (k >= per) return Tile{-1, 0, 0};
        while (g0 + k >= at + nt) {
            at += nt;
            if (++c >= a.C) return Tile{-1, 0, 0};
            len = cell_len(a, c), nt = tile_count(scored(a, c));
        }
        return Tile{c, g0 + k - at, len};
    };
    const auto pages = [&](const Tile &z, int (&pg)[4]) {
#pragma unroll
        for (int x = 0; x < 4; ++x) pg[x] = page_of(a, a.table + (int64_t)z.c * a.W, z.c >= 0 ? z.len : 0, z.t, x);
    };
    const auto old_score = [&](const Tile &z) {
        const int j = z.t * TT + lane;
        return a.earlier && j < z.len && j < a.n ? a.earlier[z.c * a.n + j] : 0.f;
    };
    Tile z = take();
    if (z.c < 0) return;
    int pg[4], pn[4];
    pages(z, pg);
    float old = old_score(z);
    Keys<DP, false> kr;
    kr.load(a, z.t, pg, lane);
    Tile next = take();
    pages(next, pn);
    while (z.c >= 0) {
        const int cell = z.c, seq = cell / a.Hkv, h = cell % a.Hkv;
        const float sl2 = (a.scale ? a.scale[h] : (float)(1.0 / sqrt((double)a.d))) * SLOG2E;
        bf16x8 q[KS][NP];
        f32x4 l;
        int hid[4];
        const T *p = (const T *)a.q + seq * a.q_seq + (tl / a.G) * a.q_tok + (h * a.G + tl % a.G) * a.q_head;
#pragma unroll
        for (int y = 0; y < KS; ++y) load_row<T, NP>(a, p, tl < a.R, Keys<DP, false>::column(y, g), q[y]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * g + i;
            l[i] = r < a.R ? a.lse[((int64_t)seq * a.T + r / a.G) * a.Hkv * a.G + h * a.G + r % a.G] * SLOG2E : INFINITY;
            hid[i] = r < a.R ? z.len - (a.T - 1 - r / a.G) : 0;
        }
        do {
            float f[4], sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 4; ++x) f[x] = sl2 * exp2_of_byte(kr.e[x]);
            f32x4 s[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                s[x] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int y = 0; y < KS; ++y) {
                    const bf16x8 kk = widen(kr.k[x][2 * y], kr.k[x][2 * y + 1]);
#pragma unroll
                    for (int u = NP - 1; u >= 0; --u) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[y][u], kk, s[x], 0, 0, 0);
                }
            }
            // the next tile: what is added to before the keys, whose use waits for all loads before
            const Tile now = z;
            const int from[4] = {pg[0], pg[1], pg[2], pg[3]};
            const float was = old;
            z = next;
#pragma unroll
            for (int x = 0; x < 4; ++x) pg[x] = pn[x];
            if (z.c >= 0) {
                old = old_score(z);
                kr.load(a, z.t, pg, lane);
                next = take();
                pages(next, pn);
            }
            const int tok = now.t * TT;
            if (tok > now.len - (a.T - 1) - TT) add_weights<true>(s, l, f, hid, tok + tl, sum);
            else add_weights<false>(s, l, f, hid, tok + tl, sum);
            put_scores(a, now.c * a.n + tok + lane, sum, from, lane, tok + lane < now.len && tok + lane < a.n, mean, was);
        } while (z.c == cell);
    }
}

// NW waves; LDS: rows as MFMA operands [row tile][key step][part][lane], their lse (base 2), and how many of the last
// tokens each does not see.
template <typename T, int DP, int NW>
__global__ void __launch_bounds__(64 * NW, DP <= 128 ? 4 : NW / 4) many_rows(ScoreArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, KS = DP / 32, NT = 64 * NW;
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tl = lane & 15, g = lane >> 4;
    bf16x8 *const qs = (bf16x8 *)lds;
    float *const ls = (float *)(lds + (size_t)a.turn * KS * NP * 64);
    int *const back = (int *)(ls + a.turn);
    int2 found[1];
    int per;
    find_shares<NT, 1, kFill>(a, gridDim.x, kManyLeast, found, &per);
    int c = __builtin_amdgcn_readfirstlane(found[0].x), at = __builtin_amdgcn_readfirstlane(found[0].y);
    if (c < 0) return;
    const int g0 = blockIdx.x * per, g1 = g0 + per;
    const float mean = 1.f / a.R, inv_g = 1.f / a.G;

    for (; c < a.C && at < g1; ++c) {
        const int len = cell_len(a, c), n = scored(a, c), nt = tile_count(n);
        const int t0 = max(g0 - at, 0), t1 = min(g1 - at, nt);
        at += nt > 0 ? nt + kFill : 0;
        if (t0 >= t1) continue;
        const int seq = c / a.Hkv, h = c % a.Hkv;
        const int32_t *row = a.table + (int64_t)c * a.W;
        const float sl2 = (a.scale ? a.scale[h] : (float)(1.0 / sqrt((double)a.d))) * SLOG2E;
        const int full = len - (a.T - 1);  // tokens that every row sees
        for (int r0 = 0; r0 < a.R; r0 += a.turn) {
            const int rows = min(a.turn, a.R - r0), tiles = (rows + 15) / 16;
            const float *before = r0 > 0 ? a.scores : a.earlier;
            int pg[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) pg[x] = page_of(a, row, t0 + w < t1 ? len : 0, t0 + w, x);
            __syncthreads();  // the rows before are done with
            constexpr int FL = NP == 1 ? 4 : 2;  // pieces of eight columns in flight
            for (int i0 = tid; i0 < tiles * KS * 64; i0 += FL * NT) {
                bf16x8 z[FL][NP];
#pragma unroll
                for (int u = 0; u < FL; ++u) {
                    const int i = i0 + u * NT, y = (i >> 6) % KS, r = r0 + 16 * ((i >> 6) / KS) + tl;
                    // row r is head r % G of position r / G; exact, since R <= 4096
                    const int pos = (int)((r + 0.5f) * inv_g), head = h * a.G + r - pos * a.G;
                    const T *p = (const T *)a.q + seq * a.q_seq + pos * a.q_tok + head * a.q_head;
                    load_row<T, NP>(a, p, r < a.R && i < tiles * KS * 64, Keys<DP, true>::column(y, g), z[u]);
                }
#pragma unroll
                for (int u = 0; u < FL; ++u) {
                    const int i = i0 + u * NT;
                    if (i < tiles * KS * 64)
#pragma unroll
                        for (int s = 0; s < NP; ++s) qs[((i >> 6) * NP + s) * 64 + lane] = z[u][s];
                }
            }
            for (int i = tid; i < 16 * tiles; i += NT) {
                const int r = r0 + i, pos = (int)((r + 0.5f) * inv_g);
                const bool in = r < a.R;
                ls[i] = in ? a.lse[((int64_t)seq * a.T + pos) * a.Hkv * a.G + h * a.G + r - pos * a.G] * SLOG2E : INFINITY;
                back[i] = in ? a.T - 1 - pos : len;
            }
            __syncthreads();
            for (int t = t0 + w; t < t1; t += NW) {
                const bool in = t * TT + lane < n;
                const int64_t out = c * a.n + t * TT + lane;
                const float old = before && in ? before[out] : 0.f;
                bf16x8 kf[4][KS];
                float f[4], sum[4] = {0.f, 0.f, 0.f, 0.f};
                {
                    Keys<DP, true> kr;
                    kr.load(a, t, pg, lane);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        f[x] = sl2 * exp2_of_byte(kr.e[x]);
#pragma unroll
                        for (int y = 0; y < KS; ++y) kf[x][y] = widen(kr.k[x][2 * y], kr.k[x][2 * y + 1]);
                    }
                }
                const int now[4] = {pg[0], pg[1], pg[2], pg[3]};
#pragma unroll
                for (int x = 0; x < 4; ++x) pg[x] = page_of(a, row, t + NW < t1 ? len : 0, t + NW, x);
                const auto all_rows = [&](auto masked) {
#pragma unroll 1
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
                        int hid[4] = {0, 0, 0, 0};
                        if constexpr (masked) {
                            const int4 b = *(const int4 *)(back + 16 * rt + 4 * g);
                            hid[0] = len - b.x, hid[1] = len - b.y, hid[2] = len - b.z, hid[3] = len - b.w;
                        }
                        add_weights<masked>(s, l, f, hid, t * TT + tl, sum);
                    }
                };
                if (t * TT > full - TT) all_rows(std::true_type());
                else all_rows(std::false_type());
                put_scores(a, out, sum, now, lane, in, mean, old);
            }
        }
    }
}

template <typename T, int DP>
hipError_t launch_scores_width(ScoreArgs &a, hipStream_t st) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;
    const int64_t tiles = a.C * ((std::min<int64_t>((int64_t)a.W << a.shift, a.n) + TT - 1) / TT);
    if (a.R <= 16) {
        constexpr int FW = DP <= (sizeof(T) == 2 ? 128 : 64) ? 16 : 8;
        hipLaunchKernelGGL((few_rows<T, DP, FW>), dim3((unsigned)std::min<int64_t>(kFewGroups, tiles)), dim3(64 * FW), 0, st, a);
        return hipGetLastError();
    }
    const int row = 2 * DP * NP;
    const auto many = [&](auto kernel, int waves, int groups, int bytes) {
        a.turn = std::min((a.R + 15) / 16 * 16, bytes / row / 16 * 16);
        const int64_t most = (tiles + kManyLeast - 1) / kManyLeast;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(groups, most)), dim3(64 * waves), (size_t)a.turn * (row + 8), st, a);
    };
    // Eight waves share rows best (256 cells of 3000 to 30000 tokens, 256 rows: 135 us, by four 150), as long as a tile's keys
    // fit their registers (64 cells of 4000 tokens, 128 rows: 192 columns 26 us by four, 56 by eight; 256 columns 32 and 103).
    constexpr int NW = DP <= 128 ? 8 : 4;
    if ((a.R + 15) / 16 * 16 * row <= kQBytes) many(many_rows<T, DP, NW>, NW, kManyGroups, kQBytes);
    else many(many_rows<T, DP, 2 * NW>, 2 * NW, kManyGroups / 2, 2 * kQBytes);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// select
//
// A cell's tokens by their scores' keys (an order of unsigned words): the key of
// the last one that stays is found digit by digit, 11, 11 and 10 bits from the
// top, by a histogram in LDS and the bin in which the rank falls; a bin that is
// taken whole ends the search.  Then the tokens above it and the first of those
// at it are written in their order, places from sums over lanes, waves and
// fours.  Scores are read once, into registers.
//
// Nothing but latency bounds it: 256 cells of 3000 to 30000 tokens, 6.5 MB, take
// 18 us, a chain of loads, six sums over a workgroup and three histograms.
//
// Rows of up to kAlone tokens: a workgroup to a cell, 256 threads where they
// hold it (2000 cells of 1000: 13 us, by 1024 threads 39; of 4000: 22 and 41).
// Longer ones in slices of 8192 tokens: a launch for each digit, in which the
// slices' histograms meet in the cell's, and one that writes.  What a slice's
// tokens above and at the key come to is read off its histogram of the last
// digit, so each slice finds its place from those of the slices before it.  (8
// cells of 131072: 27 us, by one workgroup each 187.  Slices for shorter rows too:
// 8 cells of 30000 25 us instead of 17, 256 of them 57 instead of 20.)  The row's
// width decides, since lengths are on the device: 256 cells of 3000 tokens take 135
// us in rows of 131072 and 11 in rows of 3000.
// ---------------------------------------------------------------------------
constexpr int LT = 1024;          // threads of a workgroup; fewer for short rows
constexpr int kBins = 2048;
constexpr int kAlone = 32 * LT;   // tokens of a cell that one workgroup takes alone
// tokens of a slice otherwise, and how many slices are many, so that each takes twice as many (256 cells of 131072: 176 us,
// at 8192 193, at 32768 180; 8 of them 27 at 8192, 30 at 16384)
constexpr int kSlice = 8 * LT;
constexpr int kManySlices = 256;
// Scores have few exponents, so lanes meet in a bin: each has four places (256 cells of 30000 equal scores 34 us, with one
// place 89; different ones 20 and 19).  256 threads do with one, which leaves room for more workgroups (2000 cells of 1000
// different scores 13 us, with four 22; equal ones 33 and 31).
constexpr int kCopies = 4;

struct SelectArgs {
    int64_t C, n, n_kept;
    const float *scores;
    const int32_t *lens, *keep;
    int64_t recent;
    int64_t *offsets;
    int32_t *kept_pos;
    // slices
    int slices;
    uint32_t *hist;   // [C][3][kBins]
    uint2 *state;     // [C][3] the key's digits so far, and its rank among the tokens that share them
    uint32_t *last;   // [C][slices][kBins / 2] the last digit's, of a slice
    uint32_t *above;  // [C][slices] tokens above the first two digits
};

__device__ __forceinline__ uint32_t rank_key(float x) { return x != x ? 0xFFFFFFFFu : ord_key(x); }
__device__ __forceinline__ int kept_of(const SelectArgs &a, int64_t c, int *len) {
    const int64_t l = a.lens[c];
    const int n = l < 0 ? 0 : l > a.n ? (int)a.n : (int)l, k = a.keep[c];
    *len = n;
    return k < 0 ? 0 : k > n ? n : k;
}
struct CellChoice {
    int nf, need, certain;  // tokens to choose from, how many of them, those kept in any case
};
__device__ __forceinline__ CellChoice choice_of(const SelectArgs &a, int64_t c) {
    int len;
    const int keep = kept_of(a, c, &len);
    CellChoice x;
    x.certain = (int)(a.recent < keep ? a.recent : keep);
    x.nf = len - x.certain, x.need = keep - x.certain;
    return x;
}

// Inclusive sum over the lanes up to this one: within rows of 16 by shifts, then the last lanes of the rows before.
__device__ __forceinline__ uint32_t lanes_upto(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast 31 to rows 2 and 3
    return x;
}
__device__ __forceinline__ int64_t lanes_upto(int64_t x) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t y = __shfl_up((long long)x, off);
        if ((int)(threadIdx.x & 63) >= off) x += y;
    }
    return x;
}

// Exclusive sum over the threads, and the total.
template <int NT, typename V>
__device__ __forceinline__ V scan_before(V v, V *red, V *total) {
    const int w = threadIdx.x >> 6;
    const V x = lanes_upto(v);
    if ((threadIdx.x & 63) == 63) red[w] = x;
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

// The bin from the top that holds the rem-th entry, the entries above it and its own; `count` gives a bin's entries.
struct Bin {
    uint32_t bin, above, own;
};
template <int NT, typename Count>
__device__ __forceinline__ Bin pick_bin(const Count &count, uint32_t rem, uint32_t *red, Bin *found) {
    constexpr int N = kBins / NT;  // of a thread, from the top
    uint32_t h[N], sum = 0, all;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        h[i] = count(kBins - 1 - N * (int)threadIdx.x - i);
        sum += h[i];
    }
    uint32_t before = scan_before<NT, uint32_t>(sum, red, &all);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (before < rem && rem <= before + h[i]) *found = Bin{kBins - 1 - N * threadIdx.x - i, before, h[i]};
        before += h[i];
    }
    __syncthreads();
    return *found;
}

__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_mask(int pass) { return pass == 2 ? 1023u : 2047u; }

// Scores of tokens first + 4 NT k + 4 t + i, and their keys in these scores' place; those at nf and past it get 0, which is
// below every score's key.
template <int NT, int E>
__device__ __forceinline__ void load_scores(const float *row, int first, int nf, float (&x)[E]) {
    const bool wide = ((uintptr_t)row & 15) == 0;
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
        const int j = first + 4 * NT * k + 4 * (int)threadIdx.x;
        float4 z = {0.f, 0.f, 0.f, 0.f};
        if (wide && j + 4 <= nf) {
            z = *(const float4 *)(row + j);
        } else {
            if (j < nf) z.x = row[j];
            if (j + 1 < nf) z.y = row[j + 1];
            if (j + 2 < nf) z.z = row[j + 2];
            if (j + 3 < nf) z.w = row[j + 3];
        }
        x[4 * k] = z.x, x[4 * k + 1] = z.y, x[4 * k + 2] = z.z, x[4 * k + 3] = z.w;
    }
}
template <int NT, int E>
__device__ __forceinline__ void make_keys(const float (&x)[E], int first, int nf, uint32_t (&u)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) u[i] = first + 4 * NT * (i / 4) + 4 * (int)threadIdx.x + i % 4 < nf ? rank_key(x[i]) : 0u;
}

// A histogram has CP places for each bin, one for every CP-th lane.
template <int CP, int E>
__device__ __forceinline__ void count_digit(const uint32_t (&u)[E], uint32_t key, uint32_t mask, int pass, uint32_t *hist) {
    uint32_t *mine = hist + (threadIdx.x & (CP - 1));
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (u[i] && (u[i] & mask) == key) atomicAdd(&mine[((u[i] >> digit_shift(pass)) & digit_mask(pass)) * CP], 1u);
}
template <int CP>
__device__ __forceinline__ uint32_t bin_of(const uint32_t *hist, int bin) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < CP; ++i) n += hist[bin * CP + i];
    return n;
}
template <int NT, int CP>
__device__ __forceinline__ void clear_bins(uint32_t *hist) {
#pragma unroll
    for (int i = 0; i < kBins * CP / 4; i += NT) *(uint4 *)(hist + 4 * (i + threadIdx.x)) = make_uint4(0u, 0u, 0u, 0u);
}

// Writes the positions above the key and the first rem - eq0 of those at it, from place `at` on; eq0: those at it before.
template <int NT, int E>
__device__ __forceinline__ void write_chosen(const SelectArgs &a, const uint32_t (&u)[E], int first, uint32_t key, uint32_t rem,
                                             uint32_t eq0, int64_t at, uint32_t (*red)[NT / 64]) {
    __shared__ uint32_t totals[E / 4];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    constexpr int NW = NT / 64, N = E / 4 * NW;
    uint32_t before[E / 4];  // above the key in the low half, at it in the high one (at most 4096 each)
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
        uint32_t v = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) v += u[4 * k + i] > key ? 1u : u[4 * k + i] == key ? 0x10000u : 0u;
        const uint32_t x = lanes_upto(v);
        if (lane == 63) red[k][w] = x;
        before[k] = x - v;
    }
    __syncthreads();
    // the waves' sums of each k become what lies before each wave; the totals go behind
    if (threadIdx.x < N) {
        uint32_t *const p = &red[0][0] + threadIdx.x;
        const uint32_t v = *p;
        uint32_t x = v;
#pragma unroll
        for (int off = 1; off < NW; off <<= 1) {
            const uint32_t y = __shfl_up(x, off, NW);
            if ((lane & (NW - 1)) >= off) x += y;
        }
        *p = x - v;
        if ((lane & (NW - 1)) == NW - 1) totals[threadIdx.x / NW] = x;
    }
    __syncthreads();
    // places from `at` on, in 32 bits: a cell's tokens
    const int64_t left = a.n_kept - at;
    const int room = left < 0 ? 0 : left > INT32_MAX ? INT32_MAX : (int)left;
    int32_t *const out = a.kept_pos + at;
    uint32_t eq = eq0;
    int done = 0;
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
        const uint32_t all = totals[k], b = before[k] + red[k][w];
        if (all) {
            uint32_t e = eq + (b >> 16);
            int o = done + (int)(b & 0xFFFFu) + (int)(min(e, rem) - min(eq, rem));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool same = u[4 * k + i] == key, in = u[4 * k + i] > key || (same && e < rem);
                if (in && o < room) out[o] = first + 4 * NT * k + 4 * (int)threadIdx.x + i;
                o += in, e += same;
            }
        }
        const uint32_t upto = eq + (all >> 16);
        done += (int)(all & 0xFFFFu) + (int)(min(upto, rem) - min(eq, rem));
        eq = upto;
    }
}

// Kept tokens of the cells before c and of all.
template <int NT>
__device__ __forceinline__ int64_t kept_before(const SelectArgs &a, int64_t c, longlong2 *red, int64_t *total) {
    long long lo = 0, all = 0;
    int len;
    for (int64_t i = threadIdx.x; i < a.C; i += NT) {
        const int k = kept_of(a, i, &len);
        all += k;
        lo += i < c ? k : 0;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) lo += __shfl_xor(lo, off), all += __shfl_xor(all, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_longlong2(lo, all);
    __syncthreads();
    lo = all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) lo += red[i].x, all += red[i].y;
    *total = all;
    return lo;
}
template <int NT>
__device__ __forceinline__ void write_certain(const SelectArgs &a, const CellChoice &x, int64_t o) {
    for (int i = threadIdx.x; i < x.certain; i += NT)
        if (o + x.need + i < a.n_kept) a.kept_pos[o + x.need + i] = x.nf + i;
}
// -1 behind the last kept token, by workgroup b of nb
template <int NT>
__device__ __forceinline__ void write_rest(const SelectArgs &a, int64_t total, int64_t b, int64_t nb) {
    for (int64_t i = total + b * NT + threadIdx.x; i < a.n_kept; i += nb * NT) a.kept_pos[i] = -1;
}

// OWN: every workgroup sums the cells' counts for itself; else the offsets are there.
template <int NT, int E, bool OWN>
__global__ void __launch_bounds__(NT) select_cell(SelectArgs a) {
    constexpr int CP = NT == LT ? kCopies : 1;
    __shared__ __align__(16) uint32_t hist[kBins * CP];
    __shared__ uint32_t red[E / 4][NT / 64];
    __shared__ Bin found;
    __shared__ longlong2 sums[NT / 64];
    const int64_t c = blockIdx.x;
    const CellChoice x = choice_of(a, c);
    float s[E];
    load_scores<NT, E>(a.scores + c * a.n, 0, x.need ? x.nf : 0, s);
    int64_t total, o;
    if (OWN) {
        o = kept_before<NT>(a, c, sums, &total);
        if (threadIdx.x == 0) {
            a.offsets[c] = o;
            if (c == a.C - 1) a.offsets[a.C] = total;
        }
    } else {
        o = a.offsets[c], total = a.offsets[a.C];
    }
    write_rest<NT>(a, total, c, gridDim.x);
    write_certain<NT>(a, x, o);
    if (x.need == 0) return;
    uint32_t u[E];
    make_keys<NT, E>(s, 0, x.nf, u);
    uint32_t key = 0, mask = 0, rem = 0;  // all: every key is above 0
    if (x.need < x.nf) {
        rem = x.need;
        for (int pass = 0; pass < 3; ++pass) {
            clear_bins<NT, CP>(hist);
            __syncthreads();
            count_digit<CP>(u, key, mask, pass, hist);
            __syncthreads();
            const Bin b = pick_bin<NT>([&](int i) { return bin_of<CP>(hist, i); }, rem, red[0], &found);
            key |= b.bin << digit_shift(pass), mask |= digit_mask(pass) << digit_shift(pass), rem -= b.above;
            if (b.own == rem) {  // all of the bin: no need to part it
                --key, rem = 0;  // some score's first digits, so above 0
                break;
            }
        }
    }
    write_chosen<NT, E>(a, u, 0, key, rem, 0, o, red);
}

__device__ __forceinline__ void write_offsets(const SelectArgs &a, int64_t *red) {
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
__global__ void __launch_bounds__(LT) select_offsets(SelectArgs a) {
    __shared__ int64_t red[LT / 64];
    write_offsets(a, red);
}
// The first workgroup writes the offsets, the others clear the histograms.
__global__ void __launch_bounds__(LT) select_begin(SelectArgs a) {
    __shared__ int64_t red[LT / 64];
    if (blockIdx.x == 0) {
        write_offsets(a, red);
        return;
    }
    const int64_t n = a.C * 3 * kBins / 4;
    for (int64_t i = (int64_t)(blockIdx.x - 1) * LT + threadIdx.x; i < n; i += (int64_t)(gridDim.x - 1) * LT)
        ((uint4 *)a.hist)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// The key's digits before `pass`: those before the last of them as the launch before left them, that one from the cell's
// histogram of it.  The cell's first slice leaves them for the launch after.
__device__ __forceinline__ void key_so_far(const SelectArgs &a, int64_t c, int s, int pass, uint32_t need, uint32_t *red,
                                           Bin *found, uint32_t *key, uint32_t *mask, uint32_t *rem) {
    *key = 0, *mask = 0, *rem = need;
    if (pass == 0) return;
    const int p = pass - 1;
    if (p > 0) {
        const uint2 x = a.state[c * 3 + p - 1];
        *key = x.x, *rem = x.y;
        for (int i = 0; i < p; ++i) *mask |= digit_mask(i) << digit_shift(i);
    }
    const uint32_t *hist = a.hist + (c * 3 + p) * kBins;
    const Bin b = pick_bin<LT>([&](int i) { return hist[i]; }, *rem, red, found);
    *key |= b.bin << digit_shift(p), *mask |= digit_mask(p) << digit_shift(p), *rem -= b.above;
    if (s == 0 && threadIdx.x == 0) a.state[c * 3 + p] = make_uint2(*key, *rem);
}

template <int E>
__global__ void __launch_bounds__(LT) select_digit(SelectArgs a, int pass) {
    __shared__ __align__(16) uint32_t hist[kBins * kCopies];
    __shared__ uint32_t red[LT / 64];
    __shared__ Bin found;
    const int64_t c = blockIdx.x / a.slices;
    const int s = blockIdx.x % a.slices, first = s * E * LT;
    const CellChoice x = choice_of(a, c);
    if (first >= x.nf || x.need == 0 || x.need == x.nf) return;
    float z[E];
    uint32_t u[E], key, mask, rem;
    load_scores<LT, E>(a.scores + c * a.n, first, x.nf, z);
    clear_bins<LT, kCopies>(hist);
    key_so_far(a, c, s, pass, x.need, red, &found, &key, &mask, &rem);
    make_keys<LT, E>(z, first, x.nf, u);
    __syncthreads();
    count_digit<kCopies>(u, key, mask, pass, hist);
    if (pass == 2) {
        uint32_t more = 0, all;
#pragma unroll
        for (int i = 0; i < E; ++i) more += (u[i] & mask) > key;
        scan_before<LT, uint32_t>(more, red, &all);
        if (threadIdx.x == 0) a.above[c * a.slices + s] = all;
    }
    __syncthreads();
    uint32_t *to = a.hist + (c * 3 + pass) * kBins;
    for (int i = threadIdx.x; i < (pass == 2 ? kBins / 2 : kBins); i += LT) {
        const uint32_t n = bin_of<kCopies>(hist, i);
        if (n) atomicAdd(&to[i], n);
        if (pass == 2) a.last[(c * a.slices + s) * (kBins / 2) + i] = n;
    }
}

template <int E>
__global__ void __launch_bounds__(LT) select_write(SelectArgs a) {
    __shared__ uint32_t red[E / 4][LT / 64];
    __shared__ Bin found;
    const int64_t c = blockIdx.x / a.slices;
    const int s = blockIdx.x % a.slices, first = s * E * LT;
    int64_t o = a.offsets[c];
    write_rest<LT>(a, a.offsets[a.C], blockIdx.x, gridDim.x);
    const CellChoice x = choice_of(a, c);
    if (s == 0) write_certain<LT>(a, x, o);
    if (first >= x.nf || x.need == 0) return;
    float z[E];
    uint32_t u[E], key = 0, mask, rem = 0, eq = 0;
    load_scores<LT, E>(a.scores + c * a.n, first, x.nf, z);
    if (x.need == x.nf) {
        o += first;
    } else {
        key_so_far(a, c, 1, 3, x.need, red[0], &found, &key, &mask, &rem);
        // tokens above and at the key in the slices before
        const uint32_t bin = key & 1023u;
        uint32_t more = 0, same = 0, all;
#pragma unroll 8
        for (int i = 0; i < s; ++i) {
            const uint32_t h = a.last[(c * a.slices + i) * (kBins / 2) + threadIdx.x];
            more += threadIdx.x > bin ? h : 0u;
            same += threadIdx.x == bin ? h : 0u;
        }
        for (int i = threadIdx.x; i < s; i += LT) more += a.above[c * a.slices + i];
        scan_before<LT, uint32_t>(more, red[0], &all);
        scan_before<LT, uint32_t>(same, red[0], &eq);
        o += all + min(eq, rem);
    }
    make_keys<LT, E>(z, first, x.nf, u);
    write_chosen<LT, E>(a, u, first, key, rem, eq, o, red);
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
    const int size = dtype == FW_F32 ? 4 : 2;
    a.wide = a.d % 8 == 0 && (uintptr_t)q % 16 == 0 && q_seq * size % 16 == 0 && q_tok * size % 16 == 0 && q_head * size % 16 == 0;
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

// Cells whose counts every workgroup sums for itself, which saves a launch (300 scores each: 2000 cells 9 us, with a launch
// 11.5; 4000 cells 18 and 12.5).
constexpr int64_t kOwnSums = 2048;

static int select_slices(int64_t C, int64_t n, int *size = nullptr) {
    if (n <= kAlone) return 0;
    const int tokens = C * ((n + kSlice - 1) / kSlice) > kManySlices ? 2 * kSlice : kSlice;
    if (size) *size = tokens;
    return (int)((n + tokens - 1) / tokens);
}

size_t select_ws_bytes(int64_t C, int64_t n) {
    const int64_t slices = select_slices(C, n);
    if (!slices) return 0;
    return align_up(C * 3 * kBins * 4, 256) + align_up(C * 3 * sizeof(uint2), 256) + align_up(C * slices * (kBins / 2) * 4, 256) + align_up(C * slices * 4, 256);
}

hipError_t launch_select_cells(int64_t C, const float *scores, int64_t n, const int32_t *lens, const int32_t *keep,
                               int64_t recent, int64_t n_kept, int64_t *offsets, int32_t *kept_pos, void *ws,
                               hipStream_t st) {
    SelectArgs a{C, n, n_kept, scores, lens, keep, recent, offsets, kept_pos};
    int size = 0;
    a.slices = select_slices(C, n, &size);
    const bool own = C <= kOwnSums;
    if (a.slices) {
        char *p = (char *)ws;
        a.hist = (uint32_t *)p, p += align_up(C * 3 * kBins * 4, 256);
        a.state = (uint2 *)p, p += align_up(C * 3 * sizeof(uint2), 256);
        a.last = (uint32_t *)p, p += align_up(C * a.slices * (kBins / 2) * 4, 256);
        a.above = (uint32_t *)p;
        const dim3 grid((unsigned)(C * a.slices));
        const int64_t clears = (C * 3 * kBins / 4 + LT - 1) / LT;
        hipLaunchKernelGGL(select_begin, dim3((unsigned)std::min<int64_t>(1 + clears, 1024)), dim3(LT), 0, st, a);
        const auto run = [&](auto digit, auto write) {
            for (int pass = 0; pass < 3; ++pass) hipLaunchKernelGGL(digit, grid, dim3(LT), 0, st, a, pass);
            hipLaunchKernelGGL(write, grid, dim3(LT), 0, st, a);
        };
        if (size == kSlice) run(select_digit<kSlice / LT>, select_write<kSlice / LT>);
        else run(select_digit<2 * kSlice / LT>, select_write<2 * kSlice / LT>);
        return hipGetLastError();
    }
    if (!own) hipLaunchKernelGGL(select_offsets, dim3(1), dim3(LT), 0, st, a);
    const dim3 grid((unsigned)C);
    const auto run = [&](auto k, auto o, int threads) {
        if (own) hipLaunchKernelGGL(k, grid, dim3(threads), 0, st, a);
        else hipLaunchKernelGGL(o, grid, dim3(threads), 0, st, a);
    };
    if (n <= 1024) run(select_cell<256, 4, true>, select_cell<256, 4, false>, 256);
    else if (n <= 4096) run(select_cell<256, 16, true>, select_cell<256, 16, false>, 256);
    else if (n <= 8 * LT) run(select_cell<LT, 8, true>, select_cell<LT, 8, false>, LT);
    else if (n <= 16 * LT) run(select_cell<LT, 16, true>, select_cell<LT, 16, false>, LT);
    else run(select_cell<LT, 32, true>, select_cell<LT, 32, false>, LT);
    return hipGetLastError();
}

}  // namespace fw
