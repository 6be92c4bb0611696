// Cells that share blocks of the 8-bit cache: fw_cache_fork, fw_cache_release
// and fw_cache_compact.
//
// shared[b] counts the cells that hold block b besides its first.  A cell that
// leaves a block takes one off; who finds 0 was the last, and marks the block
// with -1.  The marked blocks go on the stack in ascending order, so the result
// does not depend on who came last: collect_blocks finds their places from how
// many each run of kRun blocks has (counted as they are marked).  Blocks that a
// call takes come from the stack as it was before, so nothing that is still
// read in a call is written in it.
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int PT = 1024;    // threads of the one workgroup that serves cells in order
constexpr int WT = 256;     // threads of the others
constexpr int kRun = 4096;  // blocks whose marks are counted together

struct PageHead {
    int64_t top, left;  // free blocks before the call, and without those it takes
    int32_t ok;
};

struct PageArgs {
    int64_t C, W, n_blocks, P, n_kept, nruns;
    int shift, bs, d, dp;
    int32_t *table, *lens, *free_list, *n_free, *shared, *refused;
    uint8_t *kc, *vc, *k_exp, *v_exp;
    const int32_t *new_len, *src, *dst, *length, *which, *kept_pos;
    const int64_t *offsets;
    // workspace
    PageHead *head;
    int32_t *counts;      // [nruns] marked blocks of each run
    int32_t *claim;       // [C] the first pair or listed cell that names a cell
    int4 *plan;           // [max(C, P)] per cell, pair or listed cell
    int32_t *rank;        // [tiles] compaction: rank among its cell's taken blocks, or -1
    uint8_t *staged, *staged_exp;  // [tiles][2][bs * dp], [tiles][2]
};

__device__ __forceinline__ int64_t length_of(const PageArgs &a, int64_t c) {
    const int64_t n = a.lens[c], most = a.W << a.shift;
    return n < 0 ? 0 : n > most ? most : n;
}
__device__ __forceinline__ int64_t nb(const PageArgs &a, int64_t n) { return (n + a.bs - 1) >> a.shift; }
__device__ __forceinline__ bool is_block(const PageArgs &a, int32_t b) { return b >= 0 && b < a.n_blocks; }
__device__ __forceinline__ int64_t free_blocks(const PageArgs &a) {
    const int64_t n = a.n_free[0];
    return n < 0 ? 0 : n > a.n_blocks ? a.n_blocks : n;
}

// Exclusive sum of one value per thread of a workgroup of NT threads, and the total.
template <int NT>
__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t *red, int64_t *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    if (lane == 63) red[w] = x;
    __syncthreads();
    int64_t before = x - v, all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        const int64_t y = red[i];
        if (i < w) before += y;
        all += y;
    }
    __syncthreads();
    *total = all;
    return before;
}

__device__ __forceinline__ void leave_block(const PageArgs &a, int32_t b) {
    if (is_block(a, b) && atomicSub(&a.shared[b], 1) == 0) atomicAdd(&a.counts[b / kRun], 1);
}

// A block's codes and exponents, by a workgroup.
__device__ __forceinline__ void copy_block(const PageArgs &a, int32_t from, int32_t to) {
    const int64_t n = (int64_t)a.bs * a.dp;
    const uint4 *k0 = (const uint4 *)(a.kc + from * n), *v0 = (const uint4 *)(a.vc + from * n);
    uint4 *k1 = (uint4 *)(a.kc + to * n), *v1 = (uint4 *)(a.vc + to * n);
    for (int i = threadIdx.x; i < n / 16; i += blockDim.x) k1[i] = k0[i], v1[i] = v0[i];
    if (threadIdx.x == 0) a.k_exp[to] = a.k_exp[from], a.v_exp[to] = a.v_exp[from];
}

// Serves `n` requests in order, each thread a run of them: need(i) blocks (0 or more) for request i, -1 for one that is
// refused in any case.  done(i, served, first): its first block's rank among those taken.  Returns how many are refused.
template <typename Need, typename Done>
__device__ __forceinline__ void serve(const PageArgs &a, int64_t n, const Need &need, const Done &done) {
    __shared__ int64_t red[PT / 64];
    __shared__ int32_t refused;
    __shared__ unsigned long long taken;
    if (threadIdx.x == 0) refused = 0, taken = 0;
    const int64_t run = (n + PT - 1) / PT, i0 = threadIdx.x * run, i1 = i0 + run < n ? i0 + run : n;
    int64_t mine = 0, all;
    for (int64_t i = i0; i < i1; ++i) {
        const int64_t x = need(i);
        mine += x > 0 ? x : 0;
    }
    int64_t at = sum_before<PT>(mine, red, &all);
    const int64_t top = free_blocks(a);
    int64_t last = 0;
    int32_t out = 0;
    for (int64_t i = i0; i < i1; ++i) {
        const int64_t x = need(i), ask = x > 0 ? x : 0;
        const bool served = x == 0 || (x > 0 && at + x <= top);
        if (served && ask) last = at + ask;
        out += !served;
        done(i, served, at);
        at += ask;
    }
    if (out) atomicAdd(&refused, out);
    if (last) atomicMax(&taken, (unsigned long long)last);  // running sums only grow
    __syncthreads();
    if (threadIdx.x == 0) {
        a.refused[0] = refused;
        a.head[0] = PageHead{top, top - (int64_t)taken, 1};
    }
}
__device__ __forceinline__ int32_t fresh_block(const PageArgs &a, int64_t top, int64_t rank) { return a.free_list[top - 1 - rank]; }

__device__ __forceinline__ void clear_counts(const PageArgs &a) {
    for (int64_t i = threadIdx.x; i < a.nruns; i += blockDim.x) a.counts[i] = 0;
}

// Marked blocks of a run onto the stack.
__global__ void __launch_bounds__(WT) collect_blocks(PageArgs a) {
    __shared__ int64_t red[WT / 64];
    const int64_t run = blockIdx.x;
    const bool last = run == a.nruns - 1;
    const int mine = a.counts[run];
    if (mine == 0 && !last) return;
    int64_t before = 0, upto;
    for (int64_t i = threadIdx.x; i < run; i += WT) before += a.counts[i];
    sum_before<WT>(before, red, &upto);
    int64_t at = a.head[0].left + upto;
    if (last && threadIdx.x == 0) {
        const int64_t n = at + mine;
        a.n_free[0] = (int32_t)(n < a.n_blocks ? n : a.n_blocks);
    }
    if (mine == 0) return;
    constexpr int E = kRun / WT;
    const int64_t b0 = run * kRun + threadIdx.x * E;
    int n = 0;
    for (int i = 0; i < E; ++i) n += b0 + i < a.n_blocks && a.shared[b0 + i] < 0;
    int64_t total;
    at += sum_before<WT>(n, red, &total);
    if (n == 0) return;
    for (int i = 0; i < E; ++i)
        if (b0 + i < a.n_blocks && a.shared[b0 + i] < 0) {
            a.shared[b0 + i] = 0;
            if (at < a.n_blocks) a.free_list[at] = (int32_t)(b0 + i);
            ++at;
        }
}

// ---------------------------------------------------------------------------
// release: plan = (blocks kept, blocks held, block for the copy or -1, served)
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(PT) release_plan(PageArgs a) {
    clear_counts(a);
    const auto cut = [&](int64_t c, int64_t *old) {
        *old = length_of(a, c);
        const int64_t n = a.new_len[c] > 0 ? a.new_len[c] : 0;
        return n < *old ? n : *old;
    };
    const int64_t top = free_blocks(a);
    const auto need = [&](int64_t c) -> int64_t {
        int64_t old;
        const int64_t n = cut(c, &old);
        if (!(n & (a.bs - 1))) return 0;
        const int32_t b = a.table[c * a.W + (n >> a.shift)];
        return is_block(a, b) && a.shared[b] > 0;
    };
    serve(a, a.C, need, [&](int64_t c, bool served, int64_t first) {
        int64_t old;
        const int64_t n = cut(c, &old), x = need(c);
        a.plan[c] = make_int4((int)nb(a, n), (int)nb(a, old), served && x ? fresh_block(a, top, first) : -1, served);
        if (served) a.lens[c] = (int32_t)n;
    });
}

__global__ void __launch_bounds__(WT) release_apply(PageArgs a) {
    const int64_t c = blockIdx.x;
    const int4 p = a.plan[c];
    if (!p.w) return;
    int32_t *row = a.table + c * a.W;
    for (int64_t j = p.x + threadIdx.x; j < p.y; j += WT) {
        leave_block(a, row[j]);
        row[j] = -1;
    }
    if (is_block(a, p.z)) {
        const int32_t b = row[p.x - 1];
        copy_block(a, b, p.z);
        __syncthreads();  // everyone has read the entry
        if (threadIdx.x == 0) {
            leave_block(a, b);
            row[p.x - 1] = p.z;
        }
    }
}

// ---------------------------------------------------------------------------
// fork: plan = (tokens or -1, block for the copy or -1)
// ---------------------------------------------------------------------------
__device__ __forceinline__ bool in_range(const PageArgs &a, int32_t c) { return c >= 0 && c < a.C; }
__device__ __forceinline__ int32_t claimed(const PageArgs &a, int32_t c) {
    return __hip_atomic_load(&a.claim[c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Who is the first of `n` to name a cell.
__device__ __forceinline__ void claim_cells(const PageArgs &a, int64_t n, const int32_t *cells) {
    for (int64_t p = threadIdx.x; p < n; p += PT)
        if (in_range(a, cells[p])) __hip_atomic_store(&a.claim[cells[p]], INT32_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int64_t p = threadIdx.x; p < n; p += PT)
        if (in_range(a, cells[p])) atomicMin(&a.claim[cells[p]], (int32_t)p);
    __syncthreads();
}

__global__ void __launch_bounds__(PT) fork_plan(PageArgs a) {
    claim_cells(a, a.P, a.dst);
    for (int64_t p = threadIdx.x; p < a.P; p += PT) {  // lengths of before the call
        const int32_t s = a.src[p], t = a.dst[p];
        int64_t n = -1;
        if (in_range(a, s) && in_range(a, t) && claimed(a, t) == p && length_of(a, t) == 0) {
            n = length_of(a, s);
            if (a.length && a.length[p] < n) n = a.length[p] > 0 ? a.length[p] : 0;
        }
        a.plan[p] = make_int4((int)n, -1, 0, 0);
    }
    __syncthreads();
    const int64_t top = free_blocks(a);
    serve(a, a.P, [&](int64_t p) -> int64_t { const int n = a.plan[p].x; return n < 0 ? -1 : (n & (a.bs - 1)) != 0; },
          [&](int64_t p, bool served, int64_t first) {
              const int n = a.plan[p].x;
              if (!served) {
                  a.plan[p].x = -1;
              } else {
                  if (n & (a.bs - 1)) a.plan[p].y = fresh_block(a, top, first);
                  a.lens[a.dst[p]] = n;
              }
          });
    if (threadIdx.x == 0) a.n_free[0] = (int32_t)a.head[0].left;  // this thread wrote it
}

__global__ void __launch_bounds__(WT) fork_apply(PageArgs a) {
    const int64_t p = blockIdx.x;
    const int4 x = a.plan[p];
    if (x.x <= 0) return;
    const int32_t *from = a.table + a.src[p] * a.W;
    int32_t *to = a.table + a.dst[p] * a.W;
    const int64_t full = x.x >> a.shift;
    for (int64_t j = threadIdx.x; j < full; j += WT) {
        const int32_t b = from[j];
        to[j] = b;
        if (is_block(a, b)) atomicAdd(&a.shared[b], 1);
    }
    if (x.x & (a.bs - 1)) {
        const int32_t b = from[full];
        if (is_block(a, b) && is_block(a, x.y)) copy_block(a, b, x.y);
        if (threadIdx.x == 0) to[full] = x.y;
    }
}

// ---------------------------------------------------------------------------
// compaction
//
// The tokens that a listed cell keeps fall into tiles of one block each.  Tile j
// of listed cell p is number offsets[p] / bs + p + j: ascending offsets leave
// room for every cell's tiles, so none needs to be counted before.
// plan = (tokens kept or -1, first tile that changes, blocks to take, first of them)
// ---------------------------------------------------------------------------
__device__ __forceinline__ int64_t cell_of(const PageArgs &a, int64_t p) { return a.which ? a.which[p] : p; }
__device__ __forceinline__ int64_t tile0(const PageArgs &a, int64_t p) { return (a.offsets[p] >> a.shift) + p; }

__global__ void __launch_bounds__(WT) compact_check(PageArgs a) {
    __shared__ int64_t red[WT / 64];
    const int64_t p = blockIdx.x, c = cell_of(a, p);
    const int64_t o = a.offsets[p], e = a.offsets[p + 1], n = e - o;
    bool bad = c < 0 || c >= a.C || o < 0 || e > a.n_kept || n < 0;
    const int64_t len = bad ? 0 : length_of(a, c);
    bad = bad || n > len;
    int64_t stay = 0;
    if (!bad)
        for (int64_t i = threadIdx.x; i < n; i += WT) {
            const int64_t x = a.kept_pos[o + i], y = i > 0 ? a.kept_pos[o + i - 1] : -1;
            bad = bad || x <= y || x >= len;
            stay += x == i;
        }
    bad = __syncthreads_or(bad);
    if (bad) {
        if (threadIdx.x == 0) a.plan[p] = make_int4(-1, 0, 0, 0);
        return;
    }
    int64_t fixed;
    sum_before<WT>(stay, red, &fixed);  // positions ascend: the tokens that stay come first
    const int32_t *row = a.table + c * a.W;
    int64_t first = fixed >> a.shift;
    if (fixed == n && (n & (a.bs - 1))) {
        const int32_t b = row[first];
        if (!is_block(a, b) || a.shared[b] <= 0) ++first;
    }
    int64_t take = 0;
    const int64_t t0 = tile0(a, p);
    for (int64_t j0 = first; j0 < nb(a, n); j0 += WT) {
        const int64_t j = j0 + threadIdx.x;
        const int32_t b = j < nb(a, n) ? row[j] : -1;
        const bool other = is_block(a, b) && a.shared[b] > 0;
        int64_t all;
        const int64_t before = sum_before<WT>(other, red, &all);
        if (j < nb(a, n)) a.rank[t0 + j] = other ? (int32_t)(take + before) : -1;
        take += all;
    }
    if (threadIdx.x == 0) a.plan[p] = make_int4((int)n, (int)first, (int)take, 0);
}

__global__ void __launch_bounds__(PT) compact_plan(PageArgs a) {
    clear_counts(a);
    if (a.which) claim_cells(a, a.P, a.which);
    bool down = false;
    for (int64_t p = threadIdx.x; p < a.P; p += PT) down = down || a.offsets[p] > a.offsets[p + 1];
    down = __syncthreads_or(down);
    serve(a, a.P,
          [&](int64_t p) -> int64_t {
              const int4 x = a.plan[p];
              if (down || x.x < 0 || (a.which && claimed(a, a.which[p]) != p)) return -1;
              return x.z;
          },
          [&](int64_t p, bool served, int64_t first) {
              if (!served) a.plan[p].x = -1;
              else a.plan[p].w = (int)first;
          });
    if (threadIdx.x == 0) a.head[0].ok = !down;
}

// The listed cell that a tile belongs to, and its number there.
__device__ __forceinline__ bool find_tile(const PageArgs &a, int64_t t, int64_t *p, int64_t *j) {
    int64_t lo = 0, hi = a.P - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (tile0(a, mid) <= t) lo = mid;
        else hi = mid - 1;
    }
    const int4 x = a.plan[lo];
    *p = lo, *j = t - tile0(a, lo);
    return x.x >= 0 && *j >= x.y && *j < nb(a, x.x);
}

// The largest finite magnitude of four codes, as a code.
__device__ __forceinline__ int top_code(uint32_t x, int top) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = (x >> (8 * i)) & 0x7F;
        top = c != 0x7F && c > top ? c : top;
    }
    return top;
}
// The least exponent byte for a magnitude `code` at exponent byte e; 0 for zero.
__device__ __forceinline__ int least_exp(int code, int e) {
    if (code == 0) return 0;
    const float v = __builtin_amdgcn_cvt_pk_f32_fp8(code, false)[0];
    int x;
    const float m = frexpf(v, &x);  // 448 = 7/8 2^9
    return x - 9 + (m > 0.875f) + e;
}
__device__ __forceinline__ uint32_t scale_codes(uint32_t c, float s) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * s, a[1] * s, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * s, b[1] * s, r, true);
}
__device__ __forceinline__ float exp_ratio(int from, int to) {  // 2^(from - to): codes that are not 0 stay in range
    const int e = from - to;
    return __uint_as_float((uint32_t)(127 + (e < -126 ? -126 : e > 127 ? 127 : e)) << 23);
}
__device__ __forceinline__ int exp_byte(uint8_t e) { return e < 1 ? 1 : e > 253 ? 253 : e; }

// One tile's keys (blockIdx.y = 0) or values to the workspace, at their new exponent.
__global__ void __launch_bounds__(WT) compact_gather(PageArgs a) {
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ int32_t blk[256];
    __shared__ int16_t off[256];
    __shared__ int16_t ex[256];
    __shared__ int red[WT / 64];
    int64_t p, j;
    if (!a.head[0].ok || !find_tile(a, blockIdx.x, &p, &j)) return;
    const bool values = blockIdx.y;
    const int tid = threadIdx.x;
    const int64_t n = a.plan[p].x, c = cell_of(a, p);
    const int m = n - (j << a.shift) < a.bs ? (int)(n - (j << a.shift)) : a.bs;
    const uint8_t *codes = values ? a.vc : a.kc, *exps = values ? a.v_exp : a.k_exp;
    if (tid < a.bs) {
        int32_t b = -1;
        int x = 0, e = 1;
        if (tid < m) {
            x = a.kept_pos[a.offsets[p] + (j << a.shift) + tid];
            b = a.table[c * a.W + (x >> a.shift)];
            if (is_block(a, b)) e = exp_byte(exps[b]);
            else b = -1;
        }
        blk[tid] = b, off[tid] = (int16_t)(x & (a.bs - 1)), ex[tid] = (int16_t)e;
    }
    __syncthreads();
    const int64_t size = (int64_t)a.bs * a.dp;
    int best = 0;
    if (!values) {
        const int per = a.dp / 16;
        for (int i = tid; i < m * per; i += WT) {
            const int t = i / per, x = i - t * per;
            uint4 y = {0u, 0u, 0u, 0u};
            if (blk[t] >= 0) y = *(const uint4 *)(codes + blk[t] * size + off[t] * a.dp + 16 * x);
            *(uint4 *)(lds + 16 * i) = y;
            best = max(best, least_exp(top_code(y.x, top_code(y.y, top_code(y.z, top_code(y.w, 0)))), ex[t]));
        }
    } else {
        const int per = a.bs / 4;
        for (int i = tid; i < a.dp * per; i += WT) {
            const int r = i / per, t = 4 * (i - r * per);
            uint32_t y = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (t + u >= m || blk[t + u] < 0) continue;
                const uint32_t z = codes[blk[t + u] * size + (int64_t)r * a.bs + off[t + u]];
                y |= z << (8 * u);
                best = max(best, least_exp(top_code(z, 0), ex[t + u]));
            }
            *(uint32_t *)(lds + 4 * i) = y;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = max(best, __shfl_xor(best, o));
    if ((tid & 63) == 0) red[tid >> 6] = best;
    __syncthreads();
    best = 1;
#pragma unroll
    for (int i = 0; i < WT / 64; ++i) best = max(best, red[i]);
    best = min(best, 253);
    uint8_t *out = a.staged + (2 * (int64_t)blockIdx.x + values) * size;
    if (tid == 0) a.staged_exp[2 * (int64_t)blockIdx.x + values] = (uint8_t)best;
    if (!values) {
        for (int i = tid; i < m * a.dp / 4; i += WT)
            ((uint32_t *)out)[i] = scale_codes(((uint32_t *)lds)[i], exp_ratio(ex[4 * i / a.dp], best));
    } else {
        const int per = a.bs / 4;
        for (int i = tid; i < a.dp * per; i += WT) {
            const int t = 4 * (i % per);
            const uint32_t x = ((uint32_t *)lds)[i];
            uint32_t y = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) y |= (scale_codes((x >> (8 * u)) & 0xFFu, exp_ratio(ex[t + u], best)) & 0xFFu) << (8 * u);
            ((uint32_t *)out)[i] = y;
        }
    }
}

// Tiles from the workspace to their blocks; the workgroups behind them give back the blocks past the cells' ends.
__global__ void __launch_bounds__(WT) compact_write(PageArgs a, int64_t tiles) {
    const int tid = threadIdx.x;
    if (!a.head[0].ok) return;
    if (blockIdx.x >= tiles) {
        if (blockIdx.y) return;
        const int64_t p = blockIdx.x - tiles;
        const int4 x = a.plan[p];
        if (x.x < 0) return;
        const int64_t c = cell_of(a, p), had = nb(a, length_of(a, c));
        int32_t *row = a.table + c * a.W;
        for (int64_t j = nb(a, x.x) + tid; j < had; j += WT) {
            leave_block(a, row[j]);
            row[j] = -1;
        }
        __syncthreads();  // everyone has read the length
        if (tid == 0) a.lens[c] = x.x;
        return;
    }
    int64_t p, j;
    if (!find_tile(a, blockIdx.x, &p, &j)) return;
    const bool values = blockIdx.y;
    const int4 x = a.plan[p];
    const int m = x.x - (j << a.shift) < a.bs ? (int)(x.x - (j << a.shift)) : a.bs;
    int32_t *entry = a.table + cell_of(a, p) * a.W + j;
    const int32_t r = a.rank[blockIdx.x];
    // where a block is taken, the entry is this tile's keys' to change; its values do not need it
    const int32_t b = r >= 0 ? fresh_block(a, a.head[0].top, x.w + r) : *entry;
    if (!is_block(a, b)) return;
    const int64_t size = (int64_t)a.bs * a.dp;
    const uint8_t *in = a.staged + (2 * (int64_t)blockIdx.x + values) * size;
    uint8_t *out = (values ? a.vc : a.kc) + b * size;
    if (!values || m == a.bs) {
        const int bytes = values ? (int)size : m * a.dp;
        for (int i = tid; i < bytes / 16; i += WT) ((uint4 *)out)[i] = ((const uint4 *)in)[i];
    } else {
        for (int i = tid; i < a.dp * m; i += WT) {
            const int y = i / m, t = i - y * m;
            out[y * a.bs + t] = in[y * a.bs + t];
        }
    }
    if (tid == 0) {
        (values ? a.v_exp : a.k_exp)[b] = a.staged_exp[2 * (int64_t)blockIdx.x + values];
        if (!values && r >= 0) {
            leave_block(a, *entry);
            *entry = b;
        }
    }
}

struct PageLayout {
    char *base;
    size_t off = 0;
    template <typename T> T *take(size_t n) {
        off = align_up(off, 256);
        T *p = base ? (T *)(base + off) : nullptr;
        off += n * sizeof(T);
        return p;
    }
};
int64_t tiles_of(int64_t P, int64_t n_kept, int block_size) { return n_kept / block_size + P; }

// kind 0: release, 1: fork, 2: compact
size_t layout(PageArgs &a, int kind, void *ws) {
    PageLayout l{(char *)ws};
    a.nruns = (a.n_blocks + kRun - 1) / kRun;
    a.head = l.take<PageHead>(1);
    if (kind != 1) a.counts = l.take<int32_t>(a.nruns);
    if (kind != 0) a.claim = l.take<int32_t>(a.C);
    a.plan = l.take<int4>(kind == 0 ? a.C : a.P);
    if (kind == 2) {
        const int64_t tiles = tiles_of(a.P, a.n_kept, a.bs);
        a.rank = l.take<int32_t>(tiles);
        a.staged_exp = l.take<uint8_t>(2 * tiles);
        a.staged = l.take<uint8_t>(2 * tiles * a.bs * a.dp);
    }
    return align_up(l.off, 256);
}

PageArgs page_args(const fw_cache &cache, const fw_cells &cells) {
    PageArgs a{};
    a.C = cells.C, a.W = cells.max_blocks, a.n_blocks = cache.n_blocks;
    a.bs = cache.block_size, a.shift = __builtin_ctz(cache.block_size), a.d = (int)cache.d, a.dp = cache_row(cache.d);
    a.table = cells.table, a.lens = cells.lens, a.free_list = cells.free_list, a.n_free = cells.n_free;
    a.shared = cells.shared;
    a.kc = cache.k, a.vc = cache.v, a.k_exp = cache.k_exp, a.v_exp = cache.v_exp;
    return a;
}
}  // namespace

size_t pages_ws_bytes(const fw_cache &cache, const fw_cells &cells, int kind, int64_t P, int64_t n_kept) {
    PageArgs a = page_args(cache, cells);
    a.P = P, a.n_kept = n_kept;
    return layout(a, kind, nullptr);
}

hipError_t launch_release(const fw_cache &cache, const fw_cells &cells, const int32_t *new_len, int32_t *refused,
                          void *ws, hipStream_t st) {
    PageArgs a = page_args(cache, cells);
    a.new_len = new_len, a.refused = refused;
    layout(a, 0, ws);
    hipLaunchKernelGGL(release_plan, dim3(1), dim3(PT), 0, st, a);
    hipLaunchKernelGGL(release_apply, dim3((unsigned)a.C), dim3(WT), 0, st, a);
    hipLaunchKernelGGL(collect_blocks, dim3((unsigned)a.nruns), dim3(WT), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_fork(const fw_cache &cache, const fw_cells &cells, int64_t P, const int32_t *src, const int32_t *dst,
                       const int32_t *length, int32_t *refused, void *ws, hipStream_t st) {
    PageArgs a = page_args(cache, cells);
    a.P = P, a.src = src, a.dst = dst, a.length = length, a.refused = refused;
    layout(a, 1, ws);
    hipLaunchKernelGGL(fork_plan, dim3(1), dim3(PT), 0, st, a);
    if (P > 0) hipLaunchKernelGGL(fork_apply, dim3((unsigned)P), dim3(WT), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_cell_compact(const fw_cache &cache, const fw_cells &cells, int64_t P, const int32_t *which,
                               const int64_t *offsets, int64_t n_kept, const int32_t *kept_pos, int32_t *refused,
                               void *ws, hipStream_t st) {
    PageArgs a = page_args(cache, cells);
    a.P = P, a.which = which, a.offsets = offsets, a.n_kept = n_kept, a.kept_pos = kept_pos, a.refused = refused;
    layout(a, 2, ws);
    const int64_t tiles = tiles_of(P, n_kept, a.bs);
    if (P > 0) hipLaunchKernelGGL(compact_check, dim3((unsigned)P), dim3(WT), 0, st, a);
    hipLaunchKernelGGL(compact_plan, dim3(1), dim3(PT), 0, st, a);
    if (P == 0) return hipGetLastError();
    hipLaunchKernelGGL(compact_gather, dim3((unsigned)tiles, 2), dim3(WT), a.bs * a.dp, st, a);
    hipLaunchKernelGGL(compact_write, dim3((unsigned)(tiles + P), 2), dim3(WT), 0, st, a, tiles);
    hipLaunchKernelGGL(collect_blocks, dim3((unsigned)a.nruns), dim3(WT), 0, st, a);
    return hipGetLastError();
}

}  // namespace fw
