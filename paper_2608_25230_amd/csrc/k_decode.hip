// Attention over the 8-bit cache (fw_cache_attention): the rows of a cell
// (T new positions x the G query heads of its key/value head) over the cell's
// cached tokens,
//
//   z_rj = scale_h 2^ek(j) <q_r, code_k(j)>,   o_r = sum_j p_rj 2^ev(j) code_v(j),
//
// p the softmax of z over the tokens that row r sees, ek and ev the exponents
// of token j's block.  Every code is read once for 16 rows of the cell or more
// (launch_rows) and is exact in bf16, so the products run on the bf16 MFMA with the codes as
// they are: the block's key scale multiplies the logits, its value scale (a
// power of two) the weights.  Float32 queries and weights are taken apart into
// three bf16 parts, which hold all 24 bits, one product for each.  The weights
// of bf16 queries take two parts: one would leave an error of 2^-8 of each
// weight, which adds a third to the output's own rounding, two leave 2^-16.
// The second part's products cost 4 to 5 % where a cell has few rows (64 cells
// of 131,000 tokens: 366 to 384 us; 512 of 800 to 10,000: 58.5 to 60) and 8 to
// 13 % at 32 or 64 rows.
//
// A wave takes 64 tokens at a time.  S^T = K Q^T on 16x16x32 MFMA: row
// m = 4 g + i of key tile t is token 16 g + 4 t + i, so after four tiles lane
// group g = l / 16 holds the weights of tokens 16 g .. 16 g + 15 of query row
// l % 16, which is the order of a 16-byte piece of a value column [d][token]:
// O^T += V^T P^T takes weights and codes as they lie.  A block of 16 or more
// tokens holds a lane group's tokens whole, so scales and page numbers are one
// per lane.
//
// Cells differ in length by far, so the work is cut by length, on the device:
// all cells' tiles in a row, and kCell more for what a cell costs besides
// them, every workgroup takes the same number of them and finds from the
// lengths where it begins.  A cell that one workgroup has whole is done with
// it; the others' parts go to the workspace, joined by decode_join.
//
// Bound by HBM where there is much to read: 64 cells of 131,000 tokens, d =
// 128 (2.15 GB) in 372 to 384 us with the join, 5.6 to 5.8 TB/s; 512 cells of
// 800 to 10,000 tokens (237 MB) 60 us with the join (50 where the last-level
// cache still holds them).  More than 16 rows of a cell read it again for every
// 16, or 32 or 64 (launch_rows): 64 rows, d = 128, 64 cells of 20,000 to 33,000
// tokens 188 us, where 4 rows take 78.  8 cells of 200 to 800 tokens: 10 us,
// the launch and a chain of dependent loads (lengths, page numbers, codes).  60
// cells of up to 6000 tokens, four float32 positions: 14 us and 5.5 for the join.
// What the constants below measured, whole calls.  kWhole 8: the third case 18
// us instead of 14; 128: the fourth 34 instead of 19.  kMinTiles 16: the
// fourth 24 instead of 19; 4: the same.  kCell 0: the fourth 33 instead of 19,
// the second 63.4 instead of 60.5; 8: 20 and 61.6.
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int DW = 4;               // waves per workgroup; 8 where one takes a whole cell (kWhole)
constexpr int DT = 64;              // tokens per wave and step
constexpr int kGroups = 256;        // workgroups that share the tiles, one to a compute unit; twice that for many or narrow cells
constexpr int kMany = 256;          // cells up to which one to a compute unit is right; kManyNarrow for narrow ones
constexpr int kManyNarrow = 8;
constexpr int kMinTiles = 8;        // tiles of a workgroup at least
constexpr int kCell = 4;            // what a cell costs besides its tiles, in tiles
constexpr int kWhole = 32;          // tiles of a table row up to which a workgroup takes one cell whole
constexpr float DLOG2E = 1.4426950408889634f;
constexpr float DLN2 = 0.6931471805599453f;
constexpr float DMIN = -3.0e38f;
constexpr float DRESCALE = 8.f;

struct DecodeArgs {
    const void *q;
    int64_t q_seq, q_tok, q_head;
    int C, T, Hkv, G, W;            // cells, new positions, heads, group, blocks per table row
    int R, d;                       // rows of a cell, their width
    const uint8_t *kc, *vc, *k_exp, *v_exp;
    int64_t n_blocks;
    int shift;
    const int32_t *table, *lens;
    const float *scale;
    void *o;
    float *lse;
    int groups;                     // workgroups that share the tiles; 0: one for each cell
    bool wide;                      // 16-byte aligned queries of a multiple of 8 columns
    int2 *cells;                    // [C] first part and parts of a cell
    float *part_o, *part_lse;       // [parts][R][d], [parts][R] (base 2)
};

__device__ __forceinline__ int cell_len(const DecodeArgs &a, int c) {
    const int most = a.W << a.shift, n = a.lens[c];
    return n < 0 ? 0 : n > most ? most : n;
}

// exclusive sum of one int per thread over the workgroup
__device__ __forceinline__ int sum_before(int v, int *red, int *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    if (lane == 63) red[w] = x;
    __syncthreads();
    int before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < DW; ++i) {
        if (i < w) before += red[i];
        sum += red[i];
    }
    __syncthreads();
    *total = sum;
    return x - v + before;
}

// Tiles of a cell; an empty one has a tile too, in which nothing is seen.
__device__ __forceinline__ int tiles_of(int len) { return len > 0 ? (len + DT - 1) / DT : 1; }

// This workgroup's share of the tiles [g0, g1), the cell that holds the first and that cell's first tile; false if
// nothing is left for it.
struct Share {
    int g0, g1, cell, first, per;
};
__device__ __forceinline__ bool find_share(const DecodeArgs &a, Share *s) {
    __shared__ int red[DW], found[2];
    const int run = (a.C + 64 * DW - 1) / (64 * DW), c0 = threadIdx.x * run;
    const int c1 = c0 + run < a.C ? c0 + run : a.C;
    int mine = 0, all;
    for (int c = c0; c < c1; ++c) mine += tiles_of(cell_len(a, c)) + kCell;
    int first = sum_before(mine, red, &all);
    s->per = (all + a.groups - 1) / a.groups;
    if (s->per < kMinTiles) s->per = kMinTiles;
    s->g0 = blockIdx.x * s->per;   // below 2^31: under 2^30 tiles, kCell more for 2^22 cells at most
    if (s->g0 >= all) return false;
    s->g1 = s->g0 + s->per < all ? s->g0 + s->per : all;
    if (s->g0 >= first && s->g0 < first + mine) {
        for (int c = c0; c < c1; ++c) {
            const int n = tiles_of(cell_len(a, c)) + kCell;
            if (s->g0 < first + n) {
                found[0] = c, found[1] = first;
                break;
            }
            first += n;
        }
    }
    __syncthreads();
    s->cell = __builtin_amdgcn_readfirstlane(found[0]), s->first = __builtin_amdgcn_readfirstlane(found[1]);
    return true;
}

__device__ __forceinline__ float pow2_byte(int b) { return __uint_as_float((uint32_t)(b < 1 ? 1 : b) << 23); }

// eight codes to bf16, exactly
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], e[0], e[1]};
}

// x as the sum of NP bf16 values (1: rounded; 2: to 2^-16; 3: all bits)
template <int NP>
__device__ __forceinline__ void take_apart(float x, __bf16 (&y)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        y[i] = (__bf16)x;
        x -= (float)y[i];
    }
}

template <typename T> __device__ __forceinline__ T dnarrow(float x);
template <> __device__ __forceinline__ float dnarrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t dnarrow<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// keeps the first n of a 16-byte piece's bytes
__device__ __forceinline__ uint4 first_bytes(uint4 x, int n) {
    const auto keep = [&](int at) -> uint32_t {
        const int k = n - at;
        return k >= 4 ? ~0u : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
    };
    x.x &= keep(0), x.y &= keep(4), x.z &= keep(8), x.w &= keep(12);
    return x;
}
// bytes that hold a NaN code (0x7f or 0xff) as 0xff, the others as 0
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) {
    const uint32_t t = ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    return (t >> 7) * 0xFFu;
}

template <typename T, int DP, int RT, int NW>
__global__ void __launch_bounds__(64 * NW, RT == 1 && DP <= (sizeof(T) == 4 ? 96 : 128) ? 2 : 1) decode_part(DecodeArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, NV = sizeof(T) == 4 ? 3 : 2;  // bf16 parts of queries, of weights
    constexpr int KS = DP / 32, DB = DP / 16, KB = DP / 4;  // key steps, value tiles, key bytes of a lane
    constexpr int KW = KB / 4;                               // the same in words
    constexpr bool AHEAD = NP == 1 || DP < 256;              // loads run a tile ahead, where registers hold them
    __shared__ float mrg[NW / 2][16 * RT * (DP + 2)];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rl = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.y * 16 * RT;
    Share sh;
    int len;
    if (NW == DW && a.groups > 0) {
        if (!find_share(a, &sh)) return;
        len = cell_len(a, sh.cell);
    } else {
        len = cell_len(a, blockIdx.x);
        sh.cell = blockIdx.x, sh.first = sh.g0 = 0, sh.per = sh.g1 = tiles_of(len);
    }
    for (int c = sh.cell, first = sh.first;;) {
    const int nt = tiles_of(len), t0 = sh.g0 > first ? sh.g0 - first : 0, t1 = sh.g1 - first < nt ? sh.g1 - first : nt;
    const bool whole = t0 == 0 && t1 == nt;
    const bool last = first + nt + kCell >= sh.g1 || c + 1 >= a.C;
    const int next_len = last ? 0 : cell_len(a, c + 1);
    if (t0 == 0 && a.groups > 0 && threadIdx.x == 0 && blockIdx.y == 0)   // parts are numbered by workgroup and cell together
        a.cells[c] = make_int2(blockIdx.x + c, whole ? 1 : (first + nt - 1) / sh.per - (int)blockIdx.x + 1);
    if (NW != DW || t0 < t1) {  // else the share begins behind the cell's tiles
    const int seq = c / a.Hkv, h = c % a.Hkv;
    const int32_t *row = a.table + (int64_t)c * a.W;
    const float sl2 = (a.scale ? a.scale[h] : (float)(1.0 / sqrt((double)a.d))) * DLOG2E;

    bf16x8 qf[RT][KS][NP];
    int seen[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + rl;
        const int rc = r < a.R ? r : a.R - 1, tok = rc / a.G;
        seen[rt] = len - (a.T - 1 - tok);
        const T *qp = (const T *)a.q + seq * a.q_seq + tok * a.q_tok + (h * a.G + rc % a.G) * a.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int col = KB * g + 8 * s;
            if (a.wide) {
                if constexpr (NP == 1) {
                    uint4 x = {0u, 0u, 0u, 0u};
                    if (col < a.d) x = *(const uint4 *)(qp + col);
                    qf[rt][s][0] = __builtin_bit_cast(bf16x8, x);
                } else {
                    f32x4 x = {0.f, 0.f, 0.f, 0.f}, z = x;
                    if (col < a.d) x = *(const f32x4 *)(qp + col), z = *(const f32x4 *)(qp + col + 4);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        __bf16 y[NP];
                        take_apart<NP>(j < 4 ? x[j] : z[j - 4], y);
#pragma unroll
                        for (int n = 0; n < NP; ++n) qf[rt][s][n][j] = y[n];
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 y[NP];
                    take_apart<NP>(col + j < a.d ? Elem<T>::load(qp, col + j) : 0.f, y);
#pragma unroll
                    for (int n = 0; n < NP; ++n) qf[rt][s][n][j] = y[n];
                }
            }
        }
    }
    const int fewest = len - (a.T - 1);   // tokens that every row sees
    const int bmask = (1 << a.shift) - 1;

    f32x4 acc[RT][DB];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = DMIN, l[rt] = 0.f;
#pragma unroll
        for (int n = 0; n < DB; ++n) acc[rt][n] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    // pages of this lane's key rows (group rl / 4) and of its weights and values (group g)
    const auto page = [&](int tok) -> int {
        const int b = tok < len ? row[tok >> a.shift] : -1;
        return b >= 0 && b < a.n_blocks ? b : -1;
    };
    // Loads run ahead: the next tile's keys are asked for when this tile's are used up, its values likewise,
    // and page numbers a tile before that.  Tokens past the end and bad pages read block 0, and are masked.
    __align__(16) uint32_t kr[4][KW];
    uint4 vr[DB];
    int ke, ve;  // exponent bytes of the lane's weights' block
    const auto load_keys = [&](int base, int kp, int vp) {
        // tile x of 16 rows: row rl = token 16 (rl / 4) + 4 x + rl % 4
        const int ktok = base + 16 * (rl / 4), kb = kp < 0 ? 0 : kp, vb = vp < 0 ? 0 : vp;
        const uint8_t *kp_ = a.kc + (((int64_t)kb << a.shift) + (ktok & bmask) + (rl & 3)) * DP + KB * g;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < KW; y += (KW % 4 == 0 ? 4 : 2)) {
                if constexpr (KW % 4 == 0) *(uint4 *)&kr[x][y] = *(const uint4 *)(kp_ + 4 * x * DP + 4 * y);
                else *(uint2 *)&kr[x][y] = *(const uint2 *)(kp_ + 4 * x * DP + 4 * y);
            }
        ke = a.k_exp[vb], ve = a.v_exp[vb];
    };
    const auto load_values = [&](int base, int vp) {
        const int vtok = base + 16 * g, vb = vp < 0 ? 0 : vp;
        const uint8_t *vp_ = a.vc + (((int64_t)vb * DP + rl) << a.shift) + (vtok & bmask);
#pragma unroll
        for (int n = 0; n < DB; ++n) vr[n] = *(const uint4 *)(vp_ + ((int64_t)(16 * n) << a.shift));
    };
    const int ts = t0 + w;
    int kp = -1, vp = -1, kpn = -1, vpn = -1;
    if (AHEAD && ts < t1) {
        kp = page(ts * DT + 16 * (rl / 4)), vp = page(ts * DT + 16 * g);
        load_keys(ts * DT, kp, vp);
        load_values(ts * DT, vp);
        if (ts + NW < t1) kpn = page((ts + NW) * DT + 16 * (rl / 4)), vpn = page((ts + NW) * DT + 16 * g);
    }
    for (int t = ts; t < t1; t += NW) {
        const int base = t * DT, vtok = base + 16 * g;
        if (!AHEAD) {
            kp = page(base + 16 * (rl / 4)), vp = page(vtok);
            load_keys(base, kp, vp);
            load_values(base, vp);
        }
        const float kf = sl2 * pow2_byte(ke), vf = pow2_byte(ve);

        f32x4 s[RT][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][x] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                const bf16x8 kk = widen8(kr[x][2 * y], kr[x][2 * y + 1]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int n = NP - 1; n >= 0; --n)
                        s[rt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qf[rt][y][n], s[rt][x], 0, 0, 0);
            }
        }
        const bool more = AHEAD && t + NW < t1;
        if (more) load_keys(base + NW * DT, kpn, vpn);
        const bool masked = base + DT > fewest || __any(vp < 0);
        if (masked) {
            const int valid = vp < 0 ? 0 : len - vtok;
#pragma unroll
            for (int n = 0; n < DB; ++n) vr[n] = first_bytes(vr[n], valid);
        }
        bf16x8 pf[RT][2][NV];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int lim = vp < 0 ? 0 : seen[rt] - vtok;
            float mt = DMIN;
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[rt][x][i] *= kf;
                    if (masked && 4 * x + i >= lim) s[rt][x][i] = -INFINITY;
                    mt = fmaxf(mt, s[rt][x][i]);
                }
            mt = fmaxf(mt, __shfl_xor(mt, 16));
            mt = fmaxf(mt, __shfl_xor(mt, 32));
            const bool ask = mt > m[rt] + DRESCALE;
            if (__any(ask)) {
                // only the rows that ask for it take a new maximum: a row's bits do not depend on its neighbours
                const float mn = ask ? mt : m[rt], al = __builtin_amdgcn_exp2f(m[rt] - mn);
                m[rt] = mn;
                l[rt] *= al;
#pragma unroll
                for (int n = 0; n < DB; ++n) acc[rt][n] *= al;
            }
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(s[rt][x][i] - m[rt]);
                    sum += e;
                    __bf16 y[NV];
                    take_apart<NV>(e * vf, y);
#pragma unroll
                    for (int n = 0; n < NV; ++n) pf[rt][x / 2][n][4 * (x % 2) + i] = y[n];
                }
            l[rt] += sum;
        }
        // A row's hidden tokens have weight 0, but 0 times a NaN code is a NaN: where new positions see
        // different tokens, NaN codes go through marks of what each row sees instead.
        bool bad = false;
        if (masked && a.T > 1) {
            uint32_t e = 0;
#pragma unroll
            for (int n = 0; n < DB; ++n) e |= nan_bytes(vr[n].x) | nan_bytes(vr[n].y) | nan_bytes(vr[n].z) | nan_bytes(vr[n].w);
            bad = __any(e != 0);
        }
        if (bad) {
#pragma unroll
            for (int n = 0; n < DB; ++n) {
                const uint4 z = {nan_bytes(vr[n].x), nan_bytes(vr[n].y), nan_bytes(vr[n].z), nan_bytes(vr[n].w)};
                vr[n] = (uint4){vr[n].x & ~z.x, vr[n].y & ~z.y, vr[n].z & ~z.z, vr[n].w & ~z.w};
                const bf16x8 z0 = widen8(z.x & 0x38383838u, z.y & 0x38383838u), z1 = widen8(z.z & 0x38383838u, z.w & 0x38383838u);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int lim = vp < 0 ? 0 : seen[rt] - vtok;
                    bf16x8 y0, y1;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        y0[i] = (__bf16)(i < lim ? 1.f : 0.f);
                        y1[i] = (__bf16)(8 + i < lim ? 1.f : 0.f);
                    }
                    f32x4 u = {0.f, 0.f, 0.f, 0.f};
                    u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z0, y0, u, 0, 0, 0);
                    u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z1, y1, u, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (u[i] > 0.f) acc[rt][n][i] = __uint_as_float(0x7FC00000u);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < DB; ++n) {
            const bf16x8 v0 = widen8(vr[n].x, vr[n].y), v1 = widen8(vr[n].z, vr[n].w);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = NV - 1; x >= 0; --x) {
                    acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[rt][0][x], acc[rt][n], 0, 0, 0);
                    acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[rt][1][x], acc[rt][n], 0, 0, 0);
                }
        }
        if (more) load_values(base + NW * DT, vpn);
        kp = kpn, vp = vpn;
        const int ahead = base + 2 * NW * DT;
        kpn = vpn = -1;
        if (AHEAD && t + 2 * NW < t1) kpn = page(ahead + 16 * (rl / 4)), vpn = page(ahead + 16 * g);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16);
        l[rt] += __shfl_xor(l[rt], 32);
    }
    // join the waves, in a fixed order: the upper half writes, the lower half takes
#pragma unroll
    for (int half = NW / 2; half >= 1; half /= 2) {
        if (w >= half && w < 2 * half) {
            float *z = mrg[w - half];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                for (int n = 0; n < DB; ++n)
                    *(f32x4 *)(z + ((rt * DB + n) * 64 + lane) * 4) = acc[rt][n];
                z[16 * RT * DP + 16 * rt + rl] = m[rt];
                z[16 * RT * (DP + 1) + 16 * rt + rl] = l[rt];
            }
        }
        __syncthreads();
        if (w < half) {
            const float *z = mrg[w];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float m2 = z[16 * RT * DP + 16 * rt + rl], l2 = z[16 * RT * (DP + 1) + 16 * rt + rl];
                const float M = fmaxf(m[rt], m2);
                const float f1 = __builtin_amdgcn_exp2f(m[rt] - M), f2 = __builtin_amdgcn_exp2f(m2 - M);
                m[rt] = M;
                l[rt] = l[rt] * f1 + l2 * f2;
#pragma unroll
                for (int n = 0; n < DB; ++n) {
                    const f32x4 y = *(const f32x4 *)(z + ((rt * DB + n) * 64 + lane) * 4);
                    acc[rt][n] = acc[rt][n] * f1 + y * f2;
                }
            }
        }
        __syncthreads();
    }
    if (w == 0) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = r0 + 16 * rt + rl;
            if (r >= a.R) continue;
            const float il = l[rt] > 0.f || l[rt] != l[rt] ? 1.f / l[rt] : 0.f;
            const float lse2 = l[rt] == 0.f ? -INFINITY : m[rt] + __builtin_amdgcn_logf(l[rt]);
            const int64_t part = (int64_t)(blockIdx.x + c) * a.R + r;
            const int64_t at = (int64_t)((seq * a.T + r / a.G) * a.Hkv + h) * a.G + r % a.G;
            int d = a.d;
            asm volatile("" : "+s"(d));  // its comparisons are made here, not kept through the loop over cells
#pragma unroll
            for (int n = 0; n < DB; ++n) {
                const int col = 16 * n + 4 * g;
                if (col >= d) continue;
                const f32x4 y = acc[rt][n] * il;
                if (d % 4 == 0) {
                    if (!whole) {
                        *(f32x4 *)(a.part_o + part * a.d + col) = y;
                    } else if constexpr (NP == 3) {
                        *(f32x4 *)((T *)a.o + at * a.d + col) = y;
                    } else {
                        const bf16x4 z = {(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
                        *(bf16x4 *)((T *)a.o + at * a.d + col) = z;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (col + i >= d) continue;
                        if (whole) ((T *)a.o)[at * a.d + col + i] = dnarrow<T>(y[i]);
                        else a.part_o[part * a.d + col + i] = y[i];
                    }
                }
            }
            if (g == 0) {
                if (!whole) a.part_lse[part] = lse2;
                else if (a.lse) a.lse[at] = lse2 * DLN2;
            }
        }
    }
    }
    if (NW != DW || last) return;
    first += nt + kCell, len = next_len, ++c;
    }
}

// Joins the parts of every row whose cell has several; one wave per row: a
// lane per part for the parts' weights, then a lane per column.
template <typename T, int NC>
__global__ void __launch_bounds__(256) decode_join(DecodeArgs a) {  // NC: columns of a lane, ceil(d / 64)
    const int lane = threadIdx.x & 63;
    const int x = (int)(blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    if ((uint32_t)x >= (uint32_t)a.C * a.R) return;
    const int c = (uint32_t)x / a.R, r = (uint32_t)x % a.R;
    const int2 ci = a.cells[c];
    const int parts = __builtin_amdgcn_readfirstlane(ci.y);
    if (parts <= 1) return;
    const float *pl = a.part_lse + (int64_t)ci.x * a.R + r;
    const float *po = a.part_o + ((int64_t)ci.x * a.R + r) * a.d;
    float M = -INFINITY;
    for (int s = lane; s < parts; s += 64) M = fmaxf(M, pl[(int64_t)s * a.R]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    const float base = M == -INFINITY ? 0.f : M;
    float sum = 0.f, y[NC];
    int col[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) y[i] = 0.f, col[i] = lane + 64 * i < a.d ? lane + 64 * i : 0;
    for (int s0 = 0; s0 < parts; s0 += 64) {
        const float e = s0 + lane < parts ? pl[(int64_t)(s0 + lane) * a.R] : -INFINITY;
        const float w = __builtin_amdgcn_exp2f(e - base);
        sum += w;
        const int n = parts - s0 < 64 ? parts - s0 : 64;
#pragma unroll 8
        for (int s = 0; s < n; ++s) {
            const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
            const float *row = po + (int64_t)(s0 + s) * a.R * a.d;
#pragma unroll
            for (int i = 0; i < NC; ++i) y[i] = fmaf(ws, row[col[i]], y[i]);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    const float is = sum == 0.f ? 0.f : 1.f / sum;
    const int seq = c / a.Hkv, h = c % a.Hkv;
    const int64_t at = (int64_t)((seq * a.T + r / a.G) * a.Hkv + h) * a.G + r % a.G;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (lane + 64 * i < a.d) ((T *)a.o)[at * a.d + lane + 64 * i] = dnarrow<T>(y[i] * is);
    if (lane == 0 && a.lse) a.lse[at] = (M + (sum == 0.f ? 0.f : __builtin_amdgcn_logf(sum))) * DLN2;
}

template <typename T, int DP, int RT, int NW = DW>
void launch_part(const DecodeArgs &a, unsigned parts, hipStream_t st) {
    const dim3 grid(parts, (unsigned)((a.R + 16 * RT - 1) / (16 * RT)));
    hipLaunchKernelGGL((decode_part<T, DP, RT, NW>), grid, dim3(64 * NW), 0, st, a);
}

// Row tiles of 16 per wave: further rows of a cell go to workgroups of their
// own, which read it again.  One tile a wave leaves room for two workgroups a
// compute unit, so it is taken while the second reading comes from the
// last-level cache (256 MB), by what all tables could hold; beyond that as many
// as a wave's registers hold.  bf16, one tile / several, in us: 64 rows, d =
// 128, 8 cells of 300 to 900 tokens 15 / 22, 512 of up to 2000 (170 MB) 119 /
// 122, 512 of up to 8000 (610 MB) 478 / 348; 32 rows, d = 128, 160 MB 68 / 72,
// 600 MB 247 / 178; d = 96, 120 MB 51 / 62, 450 MB 188 / 159; d = 64, 80 MB 39 /
// 51; 64 rows, d = 64, 85 MB 68 / 84, 550 MB 367 / 321; d = 32, two tiles, 280
// MB 247 / 200 (four 273).  Two tiles at d = 64 gain nothing: 32 rows, 300 MB
// 123 / 132, 550 MB 157 / 200, 1100 MB 403 / 393.
constexpr int64_t kCached = (int64_t)256 << 20;

template <typename T, int DP>
void launch_rows(const DecodeArgs &a, unsigned parts, hipStream_t st) {
    constexpr int most = sizeof(T) == 4 || DP > 128 ? 1 : DP == 64 ? 4 : 2;
    const bool cached = ((int64_t)a.C * a.W << a.shift) * 2 * DP <= kCached;
    if (a.R <= (most == 4 ? 32 : 16) || most == 1 || cached) {
        if constexpr (DP <= (sizeof(T) == 4 ? 96 : 128)) {
            if (a.groups == 0) return launch_part<T, DP, 1, 2 * DW>(a, parts, st);
        }
        launch_part<T, DP, 1>(a, parts, st);
    } else {
        launch_part<T, DP, most>(a, parts, st);
    }
}

template <typename T>
void launch_width(const DecodeArgs &a, int dp, unsigned parts, hipStream_t st) {
    switch (dp) {
        case 32: launch_rows<T, 32>(a, parts, st); break;
        case 64: launch_rows<T, 64>(a, parts, st); break;
        case 96: launch_rows<T, 96>(a, parts, st); break;
        case 128: launch_rows<T, 128>(a, parts, st); break;
        case 192: launch_rows<T, 192>(a, parts, st); break;
        default: launch_rows<T, 256>(a, parts, st); break;
    }
}

template <typename T>
void launch_join(const DecodeArgs &a, dim3 grid, hipStream_t st) {
    switch ((a.d + 63) / 64) {
        case 1: hipLaunchKernelGGL((decode_join<T, 1>), grid, dim3(256), 0, st, a); break;
        case 2: hipLaunchKernelGGL((decode_join<T, 2>), grid, dim3(256), 0, st, a); break;
        case 3: hipLaunchKernelGGL((decode_join<T, 3>), grid, dim3(256), 0, st, a); break;
        default: hipLaunchKernelGGL((decode_join<T, 4>), grid, dim3(256), 0, st, a); break;
    }
}

// Workgroups that share the tiles, at most so many as all tables could hold work for (the lengths are on the
// device); 0 where the tables are so short that each cell has a workgroup of its own.
//
// One to a compute unit (four waves, a tile ahead) reads as fast as two where a tile is 128 columns wide or more, or
// meets more than 16 rows, and leaves half the parts to join; narrower tiles need two, except that with few cells the
// join counts for more.  256 against 512 workgroups, in us, tokens from HBM; d = 128: 8 cells of 131,000 tokens 58 / 69,
// 64 of 131,000 385 / 400, 256 of 800 to 10,000 41.7 / 40.5, 384 of those 54.9 / 52.9, 512 of them 66 / 63 (768 workgroups
// 56 and 1536 57 against 48.5 from the last-level cache).  d = 64: 8 cells of 65,000 31 / 35, 16 of 20,000 to 65,000 31 /
// 38 but of 130,000 64 / 53, 64 of 20,000 to 65,000 67 / 55, 512 of 800 to 10,000 50 / 39.
int64_t share_groups(int64_t C, int64_t R, int64_t d, int64_t W, int block_size) {
    const int64_t tiles = (W * block_size + DT - 1) / DT;
    if (tiles <= kWhole) return 0;
    const bool narrow = cache_row(d) < 128 && R <= 16;
    const int64_t groups = C > (narrow ? kManyNarrow : kMany) ? 2 * kGroups : kGroups;
    return std::min<int64_t>(groups, (C * (tiles + kCell) + kMinTiles - 1) / kMinTiles);
}
}  // namespace

size_t decode_ws_bytes(int64_t C, int64_t R, int64_t d, int64_t W, int block_size) {
    const int64_t groups = share_groups(C, R, d, W, block_size), parts = groups + C;  // a part ends with its workgroup or its cell
    return groups ? align_up(C * sizeof(int2), 256) + align_up(parts * R * d * 4, 256) + align_up(parts * R * 4, 256) : 0;
}

hipError_t launch_decode(const fw_cache &cache, int dtype, const void *q, int64_t S, int64_t T, int64_t Hq, int64_t Hkv,
                         int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table, int64_t W,
                         const int32_t *lens, const float *scale, void *o, float *lse, void *ws, hipStream_t st) {
    DecodeArgs a{};
    a.q = q, a.q_seq = q_seq, a.q_tok = q_tok, a.q_head = q_head;
    a.C = (int)(S * Hkv), a.T = (int)T, a.Hkv = (int)Hkv, a.G = (int)(Hq / Hkv), a.W = (int)W;
    a.R = a.T * a.G, a.d = (int)cache.d;
    a.kc = cache.k, a.vc = cache.v, a.k_exp = cache.k_exp, a.v_exp = cache.v_exp;
    a.n_blocks = cache.n_blocks, a.shift = __builtin_ctz(cache.block_size);
    a.table = table, a.lens = lens, a.scale = scale, a.o = o, a.lse = lse;
    const int size = dtype == FW_F32 ? 4 : 2;
    a.wide = a.d % 8 == 0 && (uintptr_t)q % 16 == 0 && q_seq * size % 16 == 0 && q_tok * size % 16 == 0 && q_head * size % 16 == 0;
    a.groups = (int)share_groups(a.C, a.R, a.d, W, cache.block_size);
    if (a.groups) {
        const int64_t parts = (int64_t)a.groups + a.C;
        char *p = (char *)ws;
        a.cells = (int2 *)p;
        p += align_up((size_t)a.C * sizeof(int2), 256);
        a.part_o = (float *)p;
        p += align_up(parts * a.R * a.d * 4, 256);
        a.part_lse = (float *)p;
    }
    const int dp = cache_row(cache.d);
    const unsigned grid = (unsigned)(a.groups ? a.groups : a.C);
    if (dtype == FW_F32) launch_width<float>(a, dp, grid, st);
    else launch_width<uint16_t>(a, dp, grid, st);
    if (a.groups) {
        const dim3 jg((unsigned)(((int64_t)a.C * a.R + 3) / 4));
        if (dtype == FW_F32) launch_join<float>(a, jg, st);
        else launch_join<uint16_t>(a, jg, st);
    }
    return hipGetLastError();
}

}  // namespace fw
