// Attention of packed prompts (fw_prompt_attention): for every query row i of
// a sequence, over the keys j of the same sequence that it sees,
//
//   z_ij = scale_h <q_i, k_j>,  m_i = max_j z_ij,  l_i = sum_j exp(z_ij - m_i),
//   o_i = sum_j exp(z_ij - m_i) v_j / l_i,   lse_i = m_i + log l_i
//
// in one pass over the keys with the running maximum and sum of the softmax
// (all exponentials base 2 on log2e-scaled logits).  A row that sees no key
// gives o = 0 and lse = -inf.
//
// The G query heads of a key/value head share its tiles: rows of a workgroup
// are (position, head of the group) pairs, position-major, so short sequences
// fill a tile G times better and a key tile is read once for all of them.
//
// Two kernels share this file: `prompt_mfma` (bf16 rows of 16-byte aligned
// strides) and `prompt_general` (any type, width and stride; float32 MFMA).
// Measured on one MI355X: 16,384 tokens, 32 query and 8 key/value heads, d =
// 128: 1.93 to 1.99 ms, 1100 to 1140 TFLOP/s of the visible pairs; 16 packed
// sequences of 66 to 4096 (some with 1777 earlier keys) 520 to 540 us, 980 to
// 1010 TFLOP/s; five float32 sequences of up to 1999, d = 80: 104 us, 74
// TFLOP/s.  A large library product reaches 1573 (bf16) and 153 (float32).
#include <type_traits>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float PLOG2E = 1.4426950408889634f;
constexpr float PLN2 = 0.6931471805599453f;
constexpr float PMIN = -3.0e38f;  // running maximum before any key (finite: differences stay defined)

struct PromptArgs {
    const void *q, *k, *v;
    int64_t Tq, Tk, B;
    int Hq, Hkv, d, G;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    const int64_t *cu_q, *cu_k;
    const float *scale;
    int causal, splits;
    void *o;          // [Tq][Hq][d] of the rows' type
    float *lse;       // [Tq][Hq] or NULL
    float *part_o;    // [splits][Tq][Hq][d] when splits > 1
    float *part_lse;  // [splits][Tq][Hq] base-2
};

// The sequence of row tile x and the tile's place in it: tiles of `rows` rows,
// the last tile of a sequence (the one that sees most keys) first.  Every wave
// takes the tiles' prefix sum over 64 sequences at a time; the result is
// wave-uniform and read into scalars.  Lengths come from the offsets clamped
// to the arrays, so no offset leads outside them.
struct Tile {
    int q0, Lq, k0, Lk;  // first query position, queries, first key, keys of the sequence
    int r0;              // first (position, head) row of the tile
};
__device__ __forceinline__ int clamp_off(int64_t x, int64_t hi) { return (int)(x < 0 ? 0 : (x > hi ? hi : x)); }
__device__ __forceinline__ int clampi(int x, int hi) { return x < 0 ? 0 : (x > hi ? hi : x); }

__device__ __forceinline__ bool find_tile(const PromptArgs &a, int x, int rows, Tile *t) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += 64) {
        const int64_t b = b0 + lane;
        int q0 = 0, n = 0, tiles = 0;
        if (b < a.B) {
            q0 = clamp_off(a.cu_q[b], a.Tq);
            n = clamp_off(a.cu_q[b + 1], a.Tq) - q0;
            if (n < 0) n = 0;
            tiles = (int)(((uint32_t)(n * a.G) + rows - 1) / rows);
        }
        int upto = tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(upto, off);
            if (lane >= off) upto += y;
        }
        upto += before;
        const unsigned long long hit = __ballot(x < upto);
        if (hit) {
            const int s = __ffsll(hit) - 1;
            t->q0 = __builtin_amdgcn_readlane(q0, s);
            t->Lq = __builtin_amdgcn_readlane(n, s);
            t->r0 = (__builtin_amdgcn_readlane(upto, s) - 1 - x) * rows;
            t->k0 = clamp_off(a.cu_k[b0 + s], a.Tk);
            const int e = clamp_off(a.cu_k[b0 + s + 1], a.Tk);
            t->Lk = e > t->k0 ? e - t->k0 : 0;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

__device__ __forceinline__ float head_scale(const PromptArgs &a, int64_t h) {
    return a.scale ? a.scale[h] : (float)(1.0 / sqrt((double)a.d));
}

template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest, ties to even
}

// ---------------------------------------------------------------------------
// General kernel: any strides, widths and both types, float32 throughout.
// Four waves of 16 rows; key tiles of 32 in LDS as float32, rows and columns
// past the sequence's end and past d as zeros; the next tile's loads fly while
// this one is computed.
//   S^T = K Q^T on v_mfma_f32_16x16x4_f32: lane l holds row l % 16, keys
//   4 (l / 16) + i of each 16-key half.  Since the order of a contraction is
//   free, lane group l / 16 takes columns 16 j + 4 (l / 16) + s at step (j, s),
//   so one 16-byte LDS read feeds four steps.
//   O^T += V^T P^T: step i takes keys 4 (l / 16) + i, which is where the
//   weights already are: they never leave their lane.
// Bound by the float32 MFMA, at 57 % of its cycles while a compute unit has
// work: chains of dependent products and LDS reads between them take the rest.
// 104 us at this tile; 64-key tiles 105 without loads that run ahead and 135
// with them (registers spill), 32-key tiles without them 109.
// ---------------------------------------------------------------------------
constexpr int GK = 32;    // keys per tile
constexpr int GR = 64;    // rows per workgroup
constexpr int GTH = 256;

// Columns c .. c + 4 of a row as float32, those past d as zeros.
template <typename T>
__device__ __forceinline__ f32x4 load4(const T *p, int c, int d, bool vec) {
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (vec) {
        if (c >= d) return y;
        if constexpr (sizeof(T) == 4) return *(const f32x4 *)(p + c);
        const uint2 w = *(const uint2 *)(p + c);
        return (f32x4){__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u)};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < d) y[i] = Elem<T>::load(p, c + i);
    return y;
}

template <typename T, int NT>
__global__ void __launch_bounds__(GTH, NT <= 5 ? 3 : 1) prompt_general(PromptArgs a, int vec) {
    constexpr int DP = 16 * NT, LD = DP + 4;
    __shared__ __align__(16) float ks[GK * LD];
    __shared__ __align__(16) float vs[GK * LD];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, rl = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.Hkv;
    const int split = blockIdx.y;
    Tile t;
    if (!find_tile(a, blockIdx.x / a.Hkv, GR, &t)) return;
    const int rows = t.Lq * a.G;
    const int r = t.r0 + 16 * w + rl;
    const bool live = r < rows;
    const int rc = live ? r : rows - 1;
    const int pos = rc / a.G, head = h * a.G + rc % a.G;
    const int64_t qrow = t.q0 + pos;
    const T *qp = (const T *)a.q + qrow * a.q_row + head * a.q_head;
    const T *kp = (const T *)a.k + t.k0 * a.k_row + h * a.k_head;
    const T *vp = (const T *)a.v + t.k0 * a.v_row + h * a.v_head;
    const float sl2 = head_scale(a, h) * PLOG2E;
    float qf[4 * NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int c = 16 * j + 4 * g + s;
            qf[4 * j + s] = c < a.d ? Elem<T>::load(qp, c) * sl2 : 0.f;
        }
    const auto sees = [&](int row) -> int {  // keys that a row sees
        return a.causal ? clampi(row / a.G + 1 - t.Lq + t.Lk, t.Lk) : t.Lk;
    };
    const int seen = sees(rc);
    const int last = t.r0 + GR < rows ? t.r0 + GR : rows;
    const int nt = (sees(last - 1) + GK - 1) / GK;
    const int j0 = (int)((int64_t)nt * split / a.splits), j1 = (int)((int64_t)nt * (split + 1) / a.splits);
    const int fewest = sees(t.r0 + 16 * w < rows ? t.r0 + 16 * w : rows - 1);  // keys that every row of the wave sees

    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = PMIN, l = 0.f;
    constexpr int CH = DP / 4, NV = (GK * CH + GTH - 1) / GTH;  // pieces of four columns, of a row and of a thread
    f32x4 kn[NV], vn[NV];
    const auto fetch = [&](int j) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int x = threadIdx.x + u * GTH, r = x / CH, c = 4 * (x % CH);
            const int64_t key = (int64_t)j * GK + r;
            kn[u] = vn[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (r < GK && key < t.Lk) {
                kn[u] = load4<T>(kp + key * a.k_row, c, a.d, vec);
                vn[u] = load4<T>(vp + key * a.v_row, c, a.d, vec);
            }
        }
    };
    if (j0 < j1) fetch(j0);
    for (int j = j0; j < j1; ++j) {
        const int key0 = j * GK;
        bool bad = false;  // an infinity or a NaN among the values
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int x = threadIdx.x + u * GTH, at = x / CH * LD + 4 * (x % CH);
            if (x >= GK * CH) break;
            *(f32x4 *)(ks + at) = kn[u];
            *(f32x4 *)(vs + at) = vn[u];
#pragma unroll
            for (int i = 0; i < 4; ++i) bad |= !(fabsf(vn[u][i]) < INFINITY);
        }
        bad = __syncthreads_or(bad);
        if (j + 1 < j1) fetch(j + 1);
        f32x4 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f32x4 kk = *(const f32x4 *)(ks + (16 * b + rl) * LD + 16 * n + 4 * g);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[x], qf[4 * n + x], s[b], 0, 0, 0);
            }
        }
        const bool masked = key0 + GK > fewest;
        if (masked) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key0 + 16 * b + 4 * g + i >= seen) s[b][i] = -INFINITY;
        }
        float mt = PMIN;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) mt = fmaxf(mt, s[b][i]);
        mt = fmaxf(mt, __shfl_xor(mt, 16));
        mt = fmaxf(mt, __shfl_xor(mt, 32));
        const float mn = fmaxf(m, mt), al = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(s[b][i] - mn);
                sum += s[b][i];
            }
        l = fmaf(l, al, sum);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] *= al;
        if (!(bad && masked)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(vs[(16 * b + 4 * g + i) * LD + 16 * n + rl], s[b][i],
                                                                      acc[n], 0, 0, 0);
        } else {
            // A hidden key's weight is 0, but 0 times an infinity or a NaN is a NaN.  The finite values go
            // through the product, and whether a row sees an infinity of either sign (or a NaN, taken as
            // both) in a column comes from products of 0 / 1 marks.
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4 up = {0.f, 0.f, 0.f, 0.f}, dn = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y = vs[(16 * b + 4 * g + i) * LD + 16 * n + rl];
                        const float sees = key0 + 16 * b + 4 * g + i < seen ? 1.f : 0.f;
                        const bool fin = fabsf(y) < INFINITY;
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(fin ? y : 0.f, s[b][i], acc[n], 0, 0, 0);
                        up = __builtin_amdgcn_mfma_f32_16x16x4f32(!fin && !(y < 0.f) ? 1.f : 0.f, sees, up, 0, 0, 0);
                        dn = __builtin_amdgcn_mfma_f32_16x16x4f32(!fin && !(y > 0.f) ? 1.f : 0.f, sees, dn, 0, 0, 0);
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[n][i] += up[i] > 0.f ? INFINITY : 0.f;
                    acc[n][i] -= dn[i] > 0.f ? INFINITY : 0.f;
                }
            }
        }
        __syncthreads();  // every wave is done with the tile
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (!live) return;
    const float il = l > 0.f || l != l ? 1.f / l : 0.f;
    const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    const int64_t orow = qrow * a.Hq + head;
    if (a.splits > 1) {
        const int64_t prow = (int64_t)split * a.Tq * a.Hq + orow;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 16 * n + 4 * g + i;
                if (c < a.d) a.part_o[prow * a.d + c] = acc[n][i] * il;
            }
        if (g == 0) a.part_lse[prow] = lse2;
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 16 * n + 4 * g + i;
                if (c < a.d) ((T *)a.o)[orow * a.d + c] = narrow<T>(acc[n][i] * il);
            }
        if (g == 0 && a.lse) a.lse[orow] = lse2 * PLN2;
    }
}

// ---------------------------------------------------------------------------
// bf16 kernel on the bf16 MFMA (d a multiple of 8 up to D, 16-byte aligned
// rows).  Four waves of 32 rows; key and value tiles of 32 rows in a ring of
// two LDS slots, filled by direct-to-LDS loads one tile ahead.
//   S^T = K Q^T on v_mfma_f32_32x32x16_bf16: lane l holds row l % 32 and keys
//   8 (i / 4) + 4 (l / 32) + i % 4, i < 16.
//   O^T += V^T P^T: since the order of a contraction is free, step kb takes
//   keys 16 kb + 4 (l / 32) + {0..3, 8..11}: the eight weights that the lane
//   already holds, rounded to bf16 in place.  V is read transposed
//   (ds_read_b64_tr_b16), four keys of one column per lane.
// The weights enter the product in bf16.  By default each is rounded once
// (relative error up to 2^-8), which puts the result about a third further from
// the exact one than its own rounding to bf16 does, and buys a third of the
// products: 16,384 tokens in 1.93 ms, 16 packed sequences 0.52.  A caller that
// wants the weights' bits asks for two parts (fine_weights; 2^-16 left of each):
// 2.85 and 0.75 ms at two workgroups a compute unit, 2.80 and 0.75 at three,
// which spill.  Either way their sum is taken in float32 before the rounding,
// so that lse keeps float32's precision.
// No maximum is taken of a tile.  The exponentials are taken from the maximum
// m so far, and only a row whose weights over the tile sum to more than GROWN
// (or to no number) takes a new one, rescales and computes the tile's weights
// again: the first tile of every row, and few after it.  bf16 keeps its
// relative precision at any such scale.
// 16-byte chunk c of row r lies at chunk c ^ k_swizzle(r) or c ^ v_swizzle(r)
// of its LDS row, so that the 16 rows of one chunk that half a wave reads of the keys,
// and the 4 rows of 4 chunks that it reads of the values, fill all 64 banks once
// (no bank conflicts counted).
//
// What bounds it: the softmax between the products.  The MFMA is busy 69 % of
// the cycles at 1.62 GHz, that of a large library product 93 % at 1.69, with
// 4.1 and 0.05 other vector instructions per MFMA one.  So what helped were fewer
// instructions per key: 32 rows a wave need 24 LDS
// reads, 16 exponentials, 16 fused multiply-adds, 16 additions and 8
// conversions for 16 products, with three workgroups of 168 registers to a
// compute unit.  On 16,384 tokens: 64-key tiles at two workgroups 2.00 to 2.07
// ms; scores, weights and values of three tiles interleaved in one wave 2.1;
// 64 rows a wave 2.5; 8 or 12 waves a workgroup 2.0 and 1.9; this 1.88.  Tiles
// in the order of their keys over all sequences were slower than sequence by
// sequence (16 packed sequences: 555 against 536 us).
// ---------------------------------------------------------------------------
constexpr int PW = 4;            // waves per workgroup
constexpr int PTH = 64 * PW;
constexpr int PR = 32 * PW;      // rows per workgroup
constexpr int PK = 32;           // keys per tile
constexpr float GROWN = 1024.f;  // a row's sum over a tile that calls for a new maximum

typedef __amdgpu_buffer_rsrc_t rsrc_t;
#define P_LDS(p) ((__attribute__((address_space(3))) void *)(p))

// Rows [0, left) of a head from base on; reads past them return zeros.
__device__ __forceinline__ rsrc_t rows_rsrc(const char *base, int64_t left, uint32_t row_bytes, int d) {
    int64_t n = left > 0 ? (left - 1) * row_bytes + 2 * d : 0;
    if (n > 0x7FFFFFFF) n = 0x7FFFFFFF;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), (short)0, (int)n, 0x00020000);
}

__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D>
__device__ __forceinline__ int k_swizzle(int r) {
    return D == 64 ? (r >> 1) & 7 : r & 15;
}
template <int D>
__device__ __forceinline__ int v_swizzle(int r) {
    return D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3);
}

// PARTS: bf16 parts of a weight
template <int D, int PARTS>
__global__ void __launch_bounds__(PTH, D == 256 ? 1 : D == 128 && PARTS == 2 ? 2 : 3) prompt_mfma(PromptArgs a) {
    constexpr int RB = 2 * D;               // bytes of an LDS row
    constexpr int TB = PK * RB;             // bytes of a tile
    constexpr int RPI = 1024 / RB;          // rows of one 64-lane load
    constexpr int TL = PK / RPI;            // loads of a tile
    constexpr int NI = (TL + PW - 1) / PW;  // of them per wave, at most
    constexpr int KS = D / 16, DB = D / 32;
    extern __shared__ __align__(1024) unsigned char psm[];
    int *bad_tile = (int *)(psm + 4 * TB);  // 1 + the last tile of each slot that holds a non-finite value
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rl = lane & 31, hh = lane >> 5;
    const int h = blockIdx.x % a.Hkv;
    const int split = blockIdx.y;
    Tile t;
    if (!find_tile(a, blockIdx.x / a.Hkv, PR, &t)) return;
    if (threadIdx.x < 2) bad_tile[threadIdx.x] = 0;
    __syncthreads();
    const int rows = t.Lq * a.G;
    const auto sees = [&](int row) -> int {  // keys that a row sees
        return a.causal ? clampi(row / a.G + 1 - t.Lq + t.Lk, t.Lk) : t.Lk;
    };
    // the lane's row (a row past the end computes the last one's and stores nothing); the copy of the lane
    // number keeps what only the masked tiles and the end need from living in registers through the loop
    const auto my_row = [&]() -> int {
        int x = threadIdx.x;
        asm volatile("" : "+v"(x));
        return t.r0 + 32 * w + (x & 31);
    };
    float sl2 = head_scale(a, h) * PLOG2E;

    // the query row; a negative scale moves into its sign, a zero one into its values
    bf16x8 qf[KS];
    {
        const int r = my_row(), rc = r < rows ? r : rows - 1;
        const uint16_t *qp = (const uint16_t *)a.q + (int64_t)(t.q0 + rc / a.G) * a.q_row + (h * a.G + rc % a.G) * a.q_head;
        const uint32_t flip = sl2 < 0.f ? 0x80008000u : 0u, keep = sl2 == 0.f ? 0u : ~0u;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int c = 16 * s + 8 * hh;
            uint4 x = {0u, 0u, 0u, 0u};
            if (c < a.d) x = *(const uint4 *)(qp + c);
            x.x = (x.x ^ flip) & keep, x.y = (x.y ^ flip) & keep, x.z = (x.z ^ flip) & keep, x.w = (x.w ^ flip) & keep;
            qf[s] = __builtin_bit_cast(bf16x8, x);
        }
        sl2 = sl2 == 0.f ? 1.f : fabsf(sl2);
    }
    const int end = t.r0 + PR < rows ? t.r0 + PR : rows;
    const int nt = (sees(end - 1) + PK - 1) / PK;
    const int j0 = (int)((int64_t)nt * split / a.splits), j1 = (int)((int64_t)nt * (split + 1) / a.splits);
    const int gfew = sees(t.r0);            // keys that every row of the workgroup sees
    const int w0 = t.r0 + 32 * w;
    const int wmost = w0 < rows ? sees(w0 + 31 < rows ? w0 + 31 : rows - 1) : 0;  // keys that some row of the wave sees

    // direct-to-LDS loads: load i of a tile fills rows RPI i .. of the slot in lane order
    const uint32_t krb = (uint32_t)(a.k_row * 2), vrb = (uint32_t)(a.v_row * 2);
    const char *kb_ = (const char *)a.k + (t.k0 * a.k_row + h * a.k_head) * 2;
    const char *vb_ = (const char *)a.v + (t.k0 * a.v_row + h * a.v_head) * 2;
    // load i: rows RPI i ..; columns past d are out of range and read zeros
    const auto offset = [&](int i, uint32_t rb, bool keys) -> uint32_t {
        const int lr = RPI * i + lane / (D / 8), c = lane % (D / 8) ^ (keys ? k_swizzle<D>(lr) : v_swizzle<D>(lr));
        return 8 * c < a.d ? (uint32_t)lr * rb + 16 * c : 0x80000000u;
    };
    const auto issue = [&](int j) {
        const int64_t key0 = (int64_t)j * PK;
        unsigned char *slot = psm + ((j - j0) & 1) * 2 * TB;
        const rsrc_t kr = rows_rsrc(kb_ + key0 * krb, t.Lk - key0, krb, a.d);
        const rsrc_t vr = rows_rsrc(vb_ + key0 * vrb, t.Lk - key0, vrb, a.d);
#pragma unroll
        for (int x = 0; x < NI; ++x) {
            const int i = w + x * PW;
            if (TL % PW && i >= TL) break;
            const uint32_t ko = offset(i, krb, true), vo = offset(i, vrb, false);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, P_LDS(slot + i * 1024), 16, ko, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, P_LDS(slot + TB + i * 1024), 16, vo, 0, 0, 0);
        }
    };
    // LDS reads: key rl, chunk 2 s + hh; value key 4 hh + (lane % 16) / 4, columns 16 ((lane / 16) % 2) + 4 (lane % 4)
    const uint32_t base = (uint32_t)(uintptr_t)P_LDS(psm);
    const uint32_t kro = base + rl * RB + ((hh ^ k_swizzle<D>(rl)) * 16);
    uint32_t vro;
    {
        const int key = 4 * hh + (lane & 15) / 4, c = 2 * ((lane >> 4) & 1) + (lane & 3) / 2;
        vro = base + TB + key * RB + ((c ^ v_swizzle<D>(key)) * 16) + 8 * (lane & 1);
    }

    f32x16 acc[DB];
#pragma unroll
    for (int n = 0; n < DB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
    float m = PMIN, l = 0.f;
    typedef __attribute__((address_space(3))) bf16x4 lds4;
    typedef __attribute__((address_space(3))) bf16x8 lds8;
    // 16 keys' values at an LDS address
    const auto value = [&](uint32_t at) __attribute__((always_inline)) -> bf16x8 {
        const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)at);
        const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)(at + 8 * RB));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // one tile of keys in the slot at `at`; masked: some row of the wave does not see all of it, the lane's
    // row sees its keys up to lim (counted from the lane's first)
    const auto step = [&](uint32_t at, int lim, auto masked) __attribute__((always_inline)) {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < KS; ++c)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(lds8 *)(uintptr_t)((kro ^ (c * 32)) + at), qf[c], s, 0, 0, 0);
        if (decltype(masked)::value) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i / 4) + i % 4 >= lim) s[i] = -INFINITY;
        }
        bf16x8 pf[2][PARTS];
        float sum;
        const auto weights = [&]() __attribute__((always_inline)) {
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -m));
                sum += p;
                pf[i / 8][0][i % 8] = (__bf16)p;
                if constexpr (PARTS == 2) pf[i / 8][1][i % 8] = (__bf16)(p - (float)pf[i / 8][0][i % 8]);
            }
        };
        weights();
        if (__any(!(sum <= GROWN))) {
            // only the rows that ask for it take a new maximum: a row's bits do not depend on its neighbours
            float mt = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
            const bool ask = half_max(sum <= GROWN ? 0.f : 1.f) > 0.f;
            const float mn = ask ? fmaxf(m, half_max(mt) * sl2) : m, al = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= al;
#pragma unroll
            for (int n = 0; n < DB; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[n][i] *= al;
            weights();
        }
        l += sum;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int n = 0; n < DB; ++n) {
                const bf16x8 v = value((vro ^ (n * 64)) + at + kb * 16 * RB);
#pragma unroll
                for (int x = PARTS - 1; x >= 0; --x) acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[kb][x], acc[n], 0, 0, 0);
            }
    };
    // A hidden key's weight is 0, but 0 times an infinity or a NaN is a NaN.  In a tile that holds such a
    // value and is hidden from some row, the value is taken out before `step`; whether a row sees an
    // infinity of either sign (or a NaN, taken as both) in a column comes from products of 0 / 1 marks, and
    // is added after it.
    uint16_t *marks = (uint16_t *)(psm + 4 * TB + 16) + threadIdx.x;
    const auto take_out = [&](uint32_t at, int lim) __attribute__((always_inline)) {
#pragma unroll 1
        for (int it = 0; it < 2 * DB; ++it) {  // column block it / 2, infinities of either sign
            const float sign = it & 1 ? -1.f : 1.f;
            f32x16 u;
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = 0.f;
#pragma unroll 1
            for (int kb = 0; kb < 2; ++kb) {
                const bf16x8 x = value((vro ^ (it / 2 * 64)) + at + kb * 16 * RB);
                bf16x8 mark, sees_;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = sign * (float)x[i];
                    mark[i] = (__bf16)(!(fabsf(y) < INFINITY) && !(y < 0.f) ? 1.f : 0.f);
                    sees_[i] = (__bf16)(16 * kb + 8 * (i / 4) + i % 4 < lim ? 1.f : 0.f);
                }
                u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mark, sees_, u, 0, 0, 0);
            }
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) bits |= u[i] > 0.f ? 1u << i : 0u;
            marks[it * PTH] = (uint16_t)bits;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < TB / 4; x += PTH) {
            uint32_t y = ((uint32_t *)(psm + at + TB))[x];
            if ((y & 0x7F80u) == 0x7F80u) y &= 0xFFFF0000u;
            if ((y & 0x7F800000u) == 0x7F800000u) y &= 0xFFFFu;
            ((uint32_t *)(psm + at + TB))[x] = y;
        }
        __syncthreads();
    };
    if (j0 < j1) issue(j0);
    int j = j0;
    // tiles that every row of the workgroup sees whole; two by two, so that the slots are constants
    const auto arrive = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // every wave's loads of this tile have landed, and every wave is done with the other slot
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (j + 1 < j1) issue(j + 1);
    };
    for (const int full = gfew / PK < j1 ? gfew / PK : j1; j < full;) {
        arrive();
        step(0, 0, std::false_type());
        if (++j >= full) break;
        arrive();
        step(2 * TB, 0, std::false_type());
        ++j;
    }
    // tiles hidden from some row
    const int mine = my_row(), seen = sees(mine < rows ? mine : rows - 1);
    for (; j < j1; ++j) {
        const int key0 = j * PK;
        const uint32_t at = ((j - j0) & 1) * 2 * TB;
        const int lim = seen - key0 - 4 * hh;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        {
            // look for non-finite values in what this wave loaded
            uint32_t e = 0;
#pragma unroll
            for (int x = 0; x < NI; ++x) {
                if (TL % PW && w + x * PW >= TL) break;
                const uint4 y = *(const uint4 *)(psm + at + TB + (x * PW + w) * 1024 + lane * 16);
                e |= ((y.x & 0x7F807F80u) + 0x00800080u) | ((y.y & 0x7F807F80u) + 0x00800080u) |
                     ((y.z & 0x7F807F80u) + 0x00800080u) | ((y.w & 0x7F807F80u) + 0x00800080u);
            }
            if (e & 0x80008000u) bad_tile[j & 1] = j + 1;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (j + 1 < j1) issue(j + 1);
        const bool bad = __builtin_amdgcn_readfirstlane(bad_tile[j & 1]) == j + 1;
        if (bad) take_out(at, lim);
        if (key0 < wmost) step(at, lim, std::true_type());
        if (bad) {
#pragma unroll
            for (int n = 0; n < DB; ++n) {
                const uint32_t up = marks[2 * n * PTH], dn = marks[(2 * n + 1) * PTH];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (up >> i & 1) acc[n][i] += INFINITY;
                    if (dn >> i & 1) acc[n][i] -= INFINITY;
                }
            }
        }
    }
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    const int r = my_row();
    if (r >= rows) return;
    const float il = l > 0.f || l != l ? 1.f / l : 0.f;
    const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    const int64_t orow = (int64_t)(t.q0 + r / a.G) * a.Hq + h * a.G + r % a.G, prow = (int64_t)split * a.Tq * a.Hq + orow;
#pragma unroll
    for (int n = 0; n < DB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 32 * n + 8 * i + 4 * hh;
            if (c >= a.d) continue;
            f32x4 y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = acc[n][4 * i + x] * il;
            if (a.splits > 1) {
                *(f32x4 *)(a.part_o + prow * a.d + c) = y;
            } else {
                bf16x4 z;
#pragma unroll
                for (int x = 0; x < 4; ++x) z[x] = (__bf16)y[x];
                *(bf16x4 *)((uint16_t *)a.o + orow * a.d + c) = z;
            }
        }
    if (hh == 0) {
        if (a.splits > 1) a.part_lse[prow] = lse2;
        else if (a.lse) a.lse[orow] = lse2 * PLN2;
    }
}

// Joins the splits of every row: o = sum_s 2^(e_s - M) o_s / sum_s 2^(e_s - M),
// M the largest e.  A thread has V columns of a row and takes four splits at a
// time, their loads in flight together, with a running maximum.  Rows outside
// the sequences stay as they are.
template <typename T, int V>
__global__ void __launch_bounds__(256) prompt_join(PromptArgs a) {
    const uint32_t per = (uint32_t)a.d / V, n = (uint32_t)(a.Tq * a.Hq);
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (x >= (int64_t)n * per) return;
    const uint32_t row = (uint32_t)(x / per), c = (uint32_t)(x - (int64_t)row * per) * V;
    const int64_t pos = row / (uint32_t)a.Hq;
    if (pos < a.cu_q[0] || pos >= a.cu_q[a.B]) return;
    float M = PMIN, sum = 0.f, y[V] = {};
    for (int s0 = 0; s0 < a.splits; s0 += 4) {
        float e[4], o[4][V];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int64_t at = (int64_t)(s0 + s < a.splits ? s0 + s : s0) * n + row;
            e[s] = a.part_lse[at];
            const float *p = a.part_o + at * a.d + c;
            if constexpr (V == 4) {
                const f32x4 w = *(const f32x4 *)p;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[s][i] = w[i];
            } else {
                o[s][0] = *p;
            }
        }
        float top = M;
#pragma unroll
        for (int s = 0; s < 4; ++s) top = fmaxf(top, e[s]);
        const float al = __builtin_amdgcn_exp2f(M - top);
        M = top, sum *= al;
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] *= al;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s0 + s >= a.splits) break;
            const float w = __builtin_amdgcn_exp2f(e[s] - M);
            sum += w;
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(w, o[s][i], y[i]);
        }
    }
    const float is = sum == 0.f ? 0.f : 1.f / sum;
    T *out = (T *)a.o + (int64_t)row * a.d + c;
    if constexpr (V == 4 && sizeof(T) == 4) {
        *(f32x4 *)out = (f32x4){y[0] * is, y[1] * is, y[2] * is, y[3] * is};
    } else if constexpr (V == 4) {
        *(bf16x4 *)out = (bf16x4){(__bf16)(y[0] * is), (__bf16)(y[1] * is), (__bf16)(y[2] * is), (__bf16)(y[3] * is)};
    } else {
        *out = narrow<T>(y[0] * is);
    }
    if (c == 0 && a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(sum)) * PLN2;
}

template <typename T>
void launch_join(const PromptArgs &a, hipStream_t st) {
    const int64_t items = a.Tq * a.Hq * (a.d % 4 == 0 ? a.d / 4 : a.d);
    const dim3 grid((unsigned)((items + 255) / 256));
    if (a.d % 4 == 0) hipLaunchKernelGGL((prompt_join<T, 4>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((prompt_join<T, 1>), grid, dim3(256), 0, st, a);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
bool prompt_fast(const fw_packed &p) {
    const auto ok = [](const void *x, int64_t row, int64_t head, int64_t d) {
        return (uintptr_t)x % 16 == 0 && row % 8 == 0 && head % 8 == 0 && row >= d && row < ((int64_t)1 << 23);
    };
    return p.dtype == FW_BF16 && p.d % 8 == 0 && ok(p.q, p.q_row, p.q_head, 0) && ok(p.k, p.k_row, p.k_head, p.d) &&
           ok(p.v, p.v_row, p.v_head, p.d);
}

int64_t row_tiles(const fw_packed &p, int rows) {  // an upper bound: the lengths are on the device
    return (p.Tq * (p.Hq / p.Hkv) + rows - 1) / rows + p.B;
}

template <int PARTS>
void launch_mfma(const PromptArgs &a, int D, dim3 grid, size_t lds, hipStream_t st) {
    if (D == 64) hipLaunchKernelGGL((prompt_mfma<64, PARTS>), grid, dim3(PTH), lds, st, a);
    else if (D == 128) hipLaunchKernelGGL((prompt_mfma<128, PARTS>), grid, dim3(PTH), lds, st, a);
    else hipLaunchKernelGGL((prompt_mfma<256, PARTS>), grid, dim3(PTH), lds, st, a);
}

template <typename T>
void launch_general(const PromptArgs &a, int vec, dim3 grid, hipStream_t st) {
    // Widths in steps that each save a quarter or more of the next instance's products: two float32 sequences of 1500,
    // 8 query and 2 key/value heads, in us: d = 32 68, 64 111, 80 138, 96 216 (266 in 128 columns), 128 272, 192 413 (531
    // in 256), 256 542.
    const int nt = (a.d + 15) / 16;
#define FW_G(n) hipLaunchKernelGGL((prompt_general<T, n>), grid, dim3(GTH), 0, st, a, vec)
    if (nt <= 2) FW_G(2);
    else if (nt <= 4) FW_G(4);
    else if (nt <= 5) FW_G(5);
    else if (nt <= 6) FW_G(6);
    else if (nt <= 8) FW_G(8);
    else if (nt <= 12) FW_G(12);
    else FW_G(16);
#undef FW_G
}
}  // namespace

// Ranges that a row's keys are split into: at most as many as fill the card
// (three workgroups to a compute unit), and of those the cheapest by the time
// of one range, and, if there is more than one, of writing and joining the
// rows' parts.  In keys of a workgroup's time (0.0215 us in the bf16 kernel,
// 0.08 in the other): a part 1 / 96 or 1 / 384, the join's launch 160 or 40.
// Taken for a sequence halfway between the average one and one that has all
// the keys, since the lengths are on the device.  One sequence, split so
// against whole, in us: bf16, d = 128, 1000 tokens, 4 heads 18.6 / 27.4, 8
// heads 21.2 / 27.6, 32 heads whole 29.4 (in two 38.1); 4096 tokens, 4 heads
// 50 / 91, 8 heads 72 / 94; float32, d = 80, 6 heads, 500 tokens 24 / 45, 2000
// 76 / 157; d = 128, 32 heads, 500 tokens 70 / 65, 1000 137 / 146.
int prompt_splits(const fw_packed &p) {
    const bool fast = prompt_fast(p);
    const int64_t tiles = row_tiles(p, fast ? PR : GR) * p.Hkv, rows = p.Tq * p.Hq;
    const int64_t fill = std::min<int64_t>((768 + tiles / 2) / (tiles > 0 ? tiles : 1), 16);
    const int64_t keys = (p.Tk / (p.B > 0 ? p.B : 1) + p.Tk) / 2;
    int64_t best = 1, least = keys;
    for (int64_t s = 2; s <= fill; ++s) {
        const int64_t cost = keys / s + rows * s / (fast ? 96 : 384) + (fast ? 160 : 40);
        if (cost < least) best = s, least = cost;
    }
    return (int)best;
}

hipError_t launch_prompt(const fw_packed &p, void *o, float *lse, int splits, float *part_o, float *part_lse,
                         hipStream_t st) {
    PromptArgs a{};
    a.q = p.q, a.k = p.k, a.v = p.v;
    a.Tq = p.Tq, a.Tk = p.Tk, a.B = p.B, a.Hq = (int)p.Hq, a.Hkv = (int)p.Hkv;
    a.d = (int)p.d, a.G = (int)(p.Hq / p.Hkv);
    a.q_row = p.q_row, a.q_head = p.q_head, a.k_row = p.k_row, a.k_head = p.k_head, a.v_row = p.v_row, a.v_head = p.v_head;
    a.cu_q = p.cu_q, a.cu_k = p.cu_k, a.scale = p.scale;
    a.causal = p.causal, a.splits = splits;
    a.o = o, a.lse = lse, a.part_o = part_o, a.part_lse = part_lse;
    if (prompt_fast(p)) {
        const dim3 grid((unsigned)(row_tiles(p, PR) * p.Hkv), (unsigned)splits);
        const int D = a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256;
        const size_t lds = (size_t)2 * 2 * PK * 2 * D + 16 + (size_t)D / 32 * 2 * 2 * PTH;  // two slots, flags, marks
        if (p.fine_weights) launch_mfma<2>(a, D, grid, lds, st);
        else launch_mfma<1>(a, D, grid, lds, st);
    } else {
        const dim3 grid((unsigned)(row_tiles(p, GR) * p.Hkv), (unsigned)splits);
        const int size = p.dtype == FW_F32 ? 4 : 2, q = 4;
        const int vec = p.d % q == 0 && p.k_row % q == 0 && p.k_head % q == 0 && p.v_row % q == 0 && p.v_head % q == 0 &&
                        (uintptr_t)p.k % (4 * size) == 0 && (uintptr_t)p.v % (4 * size) == 0;
        if (p.dtype == FW_F32) launch_general<float>(a, vec, grid, st);
        else launch_general<uint16_t>(a, vec, grid, st);
    }
    if (splits > 1) {
        if (p.dtype == FW_F32) launch_join<float>(a, st);
        else launch_join<uint16_t>(a, st);
    }
    return hipGetLastError();
}

}  // namespace fw
