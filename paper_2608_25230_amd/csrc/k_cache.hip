// The 8-bit cache's bookkeeping and its store.
//
// fw_block_tables gives cells (one sequence's key/value head) the blocks that
// their new lengths need, takes back what they no longer need, and lists the
// slot of every token that comes.  fw_cache_store rounds rows of keys and
// values to e4m3 with one power-of-two scale per block and writes them there.
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// block tables
//
// With nb(L) = ceil(L / block_size): a cell that shrinks gives back
// nb(old) - nb(new) blocks, one that grows needs nb(new) - nb(old).  Three
// running sums over the cells (blocks back, blocks needed, tokens added) fix
// every place: the r-th block given back goes to stack position
// n_free + R - 1 - r, the k-th block needed comes from top - 1 - k (top =
// n_free + R), so a return right after a growth restores the stack.  A cell
// that needs blocks is served if its running sum of needs stays within top,
// one that needs none always.
//
// tables_scan, one workgroup, takes the sums (each thread a run of cells) and
// writes lengths, offsets and sums; tables_move, over the whole card, moves
// the blocks and writes the slots.  Blocks that come back may be taken in the
// same call, so where cells shrink and grow in one call the scan moves the
// returned blocks itself.  Small calls run in the one workgroup alone, a
// cell's few blocks and slots by the thread that has its sums: a launch costs
// more than their work.
//
// Bound by chains of dependent loads and by launches.  2048 cells that grow by
// a token: 10 us on the GPU in one launch, 9 + 7.5 in two.  256 cells, 1.5 M
// slots and 23 k blocks: 6.5 + 12 us (12 MB, 2.4 us at copy rate); one workgroup
// alone would take 1.9 ms.  So one launch is for calls that list at most 8192
// slots and, where they list none and any length may go, for tables of at most
// 16,384 blocks.  A call between two events, in us: 4135 cells of 3 blocks, 748
// k slots 34 (one launch 1250); 500 cells that grow by 17 each 19.6 (32), by 15
// in one launch 21 (cells' own threads; the workgroup together 29).
//
// Where one call gives back and takes (or lists few slots), one workgroup moves
// all that comes back: with 2048 cells, 8 that end and the others growing by a
// token 27, 64 of 20,000 tokens ending 80, half of 20,000 tokens ending (281 k
// blocks) 1000; 256 of 20,000 ending while 256 begin 257, where either alone
// takes under 40.  A program that ends very many long cells at once gives them
// back in a call of its own.
// ---------------------------------------------------------------------------
constexpr int TT = 1024;  // threads of the scan

struct TableHead {
    int64_t back, take, n_free, top;  // blocks given back and taken, the stack before, the stack with what came back
};
struct TableCell {
    int32_t old_len, had, want, served;
};
struct TableArgs {
    int64_t C, W, n_blocks, n_slots;
    int shift;  // log2 of the block size
    const int32_t *old_len, *new_len;
    int32_t *table, *free_list, *n_free;
    int64_t *slots, *offsets;
    int32_t *lens, *refused;
    TableHead *head;
    TableCell *cells;              // [C]
    int64_t *back_off, *need_off;  // [C + 1] exclusive sums
};

struct CellPlan {
    int32_t o, n;
    int64_t had, want, back, need, add;
    bool fits;
};
__device__ __forceinline__ CellPlan plan_cell(const TableArgs &a, int64_t c) {
    CellPlan p;
    p.o = a.old_len[c] > 0 ? a.old_len[c] : 0;
    p.n = a.new_len[c] > 0 ? a.new_len[c] : 0;
    const int64_t up = ((int64_t)1 << a.shift) - 1;
    p.had = (p.o + up) >> a.shift;
    if (p.had > a.W) p.had = a.W;
    p.want = (p.n + up) >> a.shift;
    p.fits = p.want <= a.W;  // a length beyond the table's row is refused
    if (!p.fits) p.want = p.had;
    p.back = p.had > p.want ? p.had - p.want : 0;
    p.need = p.want > p.had ? p.want - p.had : 0;
    p.add = p.n > p.o ? (int64_t)p.n - p.o : 0;
    return p;
}

// Exclusive sums of NV values per thread over the workgroup, and their totals.
template <int NV>
__device__ __forceinline__ void block_sums(const int64_t (&v)[NV], int64_t (&before)[NV], int64_t (&total)[NV],
                                           int64_t (*red)[TT / 64]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        int64_t x = v[i];
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        if (lane == 63) red[i][w] = x;
        before[i] = x - v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        total[i] = 0;
#pragma unroll
        for (int j = 0; j < TT / 64; ++j) {
            const int64_t y = red[i][j];
            if (j < w) before[i] += y;
            total[i] += y;
        }
    }
    __syncthreads();
}

// the last c of [0, n) with off[c] <= x (off ascending, off[0] <= x)
__device__ __forceinline__ int64_t find_cell(const int64_t *off, int64_t n, int64_t x) {
    int64_t lo = 0, hi = n - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (off[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ void move_back(const TableArgs &a, const TableHead &hd, int64_t first, int64_t step) {
    for (int64_t r = first; r < hd.back; r += step) {
        const int64_t c = find_cell(a.back_off, a.C, r);
        int32_t *e = a.table + c * a.W + a.cells[c].want + (r - a.back_off[c]);
        const int64_t p = hd.n_free + hd.back - 1 - r;
        if (p < a.n_blocks) a.free_list[p] = *e;
        *e = -1;
    }
}

__device__ __forceinline__ void take_blocks(const TableArgs &a, const TableHead &hd, int64_t first, int64_t step) {
    for (int64_t k = first; k < hd.take; k += step) {
        const int64_t c = find_cell(a.need_off, a.C, k);
        a.table[c * a.W + a.cells[c].had + (k - a.need_off[c])] = a.free_list[hd.top - 1 - k];
    }
}

// The slot of a cell's token at `pos`; a new block straight off the stack, where take_blocks finds the same.
__device__ __forceinline__ int64_t slot_of(const TableArgs &a, const TableHead &hd, int64_t c, const TableCell &t, int64_t need_off,
                                           int64_t pos) {
    if (!t.served) return -1;
    const int64_t b = pos >> a.shift;
    const int32_t e = b < t.had ? a.table[c * a.W + b] : a.free_list[hd.top - 1 - (need_off + b - t.had)];
    return e < 0 ? -1 : ((int64_t)e << a.shift) + (pos & (((int64_t)1 << a.shift) - 1));
}

// four tokens' slots at a time; `offsets` may be a copy in LDS
__device__ __forceinline__ void write_slots(const TableArgs &a, const TableHead &hd, const int64_t *offsets, int64_t first,
                                            int64_t step) {
    const int64_t total = offsets[a.C], n = a.slots ? (total < a.n_slots ? total : a.n_slots) : 0;
    for (int64_t i0 = 4 * first; i0 < n; i0 += 4 * step) {
        int64_t c = find_cell(offsets, a.C, i0);
        for (int64_t i = i0; i < i0 + 4 && i < n; ++i) {
            while (i >= offsets[c + 1]) ++c;
            const TableCell t = a.cells[c];
            a.slots[i] = slot_of(a, hd, c, t, a.need_off[c], t.old_len + (i - offsets[c]));
        }
    }
}

// Blocks or tokens of a cell that its own thread moves, if no cell has more.  500 cells that grow by 15 tokens: 21 us
// against 29 by the workgroup together (8 as the limit); by 8: 17 against 21 (1 as the limit).
constexpr int kFew = 32;

template <bool ALL>
__global__ void __launch_bounds__(TT) tables_scan(TableArgs a) {
    __shared__ int64_t red[3][TT / 64];
    const int64_t run = (a.C + TT - 1) / TT, c0 = threadIdx.x * run;
    const int64_t c1 = c0 + run < a.C ? c0 + run : a.C;
    int64_t sum[3] = {0, 0, 0}, at[3], total[3];  // blocks back, blocks needed, tokens added
    bool few = true;
    for (int64_t c = c0; c < c1; ++c) {
        const CellPlan p = plan_cell(a, c);
        sum[0] += p.back, sum[1] += p.need, sum[2] += p.add;
        few = few && p.back <= kFew && p.need <= kFew && p.add <= kFew;
    }
    int64_t n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : n_free > a.n_blocks ? a.n_blocks : n_free;
    const bool direct = ALL && !__syncthreads_or(!few);
    block_sums<3>(sum, at, total, red);
    TableHead hd;
    hd.back = total[0], hd.n_free = n_free;
    hd.top = n_free + hd.back < a.n_blocks ? n_free + hd.back : a.n_blocks;
    if (threadIdx.x == 0) a.offsets[a.C] = total[2];
    int64_t take = 0, refused = 0;
    if (direct) {
        if (hd.back > 0) {
            int64_t r = at[0];
            for (int64_t c = c0; c < c1; ++c) {
                const CellPlan p = plan_cell(a, c);
                for (int64_t i = 0; i < p.back; ++i, ++r) {
                    int32_t *e = a.table + c * a.W + p.want + i;
                    if (n_free + hd.back - 1 - r < a.n_blocks) a.free_list[n_free + hd.back - 1 - r] = *e;
                    *e = -1;
                }
            }
            __syncthreads();  // blocks that came back may be taken
        }
    } else if (threadIdx.x == 0) {
        a.need_off[a.C] = total[1], a.back_off[a.C] = hd.back;
    }
    for (int64_t c = c0; c < c1; ++c) {
        const CellPlan p = plan_cell(a, c);
        const bool served = p.fits && (p.need == 0 || at[1] + p.need <= hd.top);
        const TableCell t = {p.o, (int32_t)p.had, (int32_t)p.want, served};
        a.offsets[c] = at[2];
        a.lens[c] = served ? p.n : p.o;  // may be old_len: this thread alone reads and writes the cell
        if (direct) {
            if (served)
                for (int64_t i = 0; i < p.need; ++i) a.table[c * a.W + p.had + i] = a.free_list[hd.top - 1 - (at[1] + i)];
            for (int64_t i = 0; i < p.add && at[2] + i < a.n_slots; ++i) a.slots[at[2] + i] = slot_of(a, hd, c, t, at[1], p.o + i);
        } else {
            a.cells[c] = t, a.back_off[c] = at[0], a.need_off[c] = at[1];
        }
        if (served && p.need > 0) take = at[1] + p.need;
        refused += !served;
        at[0] += p.back, at[1] += p.need, at[2] += p.add;
    }
    // running sums only grow, so what is taken is the largest served one
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int64_t y = __shfl_xor(take, off);
        take = y > take ? y : take;
        refused += __shfl_xor(refused, off);
    }
    if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = take, red[1][threadIdx.x >> 6] = refused;
    __syncthreads();  // also: the cells' records are read by every thread from here on
    refused = 0;
#pragma unroll
    for (int i = 0; i < TT / 64; ++i) {
        take = red[0][i] > take ? red[0][i] : take;
        refused += red[1][i];
    }
    hd.take = take;
    if (threadIdx.x == 0) {
        a.n_free[0] = (int32_t)(hd.top - hd.take);
        a.refused[0] = (int32_t)refused;
    }
    if (direct) return;
    const bool mine = ALL || hd.take > 0;
    if (mine && hd.back > 0) {
        move_back(a, hd, threadIdx.x, TT);
        __syncthreads();  // blocks that came back may be taken
    }
    if (ALL) {
        take_blocks(a, hd, threadIdx.x, TT);
        write_slots(a, hd, a.offsets, threadIdx.x, TT);
    } else if (threadIdx.x == 0) {
        if (mine) hd.back = 0;
        a.head[0] = hd;
    }
}

// What the scan left: returned blocks (then none is taken), or blocks taken and slots.
// Cells whose offsets are staged in LDS where slots are listed: 256 cells, 3.3 M slots 39.5 us against 45 without; 500
// cells, 8500 slots 19.6 against 21.
constexpr int kStage = 2048;
__global__ void __launch_bounds__(256) tables_move(TableArgs a) {
    __shared__ int64_t staged[kStage + 1];
    const TableHead hd = a.head[0];
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    move_back(a, hd, first, step);
    take_blocks(a, hd, first, step);
    if (a.n_slots == 0) return;
    if (a.C <= kStage) {
        for (int64_t c = threadIdx.x; c <= a.C; c += 256) staged[c] = a.offsets[c];
        __syncthreads();
        write_slots(a, hd, staged, first, step);
    } else {
        write_slots(a, hd, a.offsets, first, step);
    }
}

// ---------------------------------------------------------------------------
// the store
//
// A block's scale is 2^e, e the least exponent with amax <= 448 2^e over its
// finite values, so x 2^-e is exact and one rounding (to nearest, ties to
// even) makes the code: an e4m3 value keeps its relative precision under any
// power of two, and a block that grows takes a larger e by shifting its codes,
// which loses nothing but subnormals.  Values that are not finite become NaN.
//
// Tokens of one call that lie in consecutive slots of one block are a run,
// taken by one workgroup: the run's largest magnitude, the block's exponent
// (with what it held before, if the run does not open the block), the rows.
// Keys lie [token][d], values [d][token], the order in which the attention's
// matrix instructions take them.
//
// Bound by HBM: 1.49 M bf16 rows of 128 in 257 us, 4.64 TB/s of the bytes read
// and written (a large copy: 4.96).  Loads with branches and 64-bit addresses
// took 318 us, keys and values on workgroups of their own 480 (registers).
// Float32 rows: 396 us at d = 128, 5.0 TB/s, 275 at d = 80, 4.5.  One token for
// each of a step's cells: 9 us, launch and load latency.
//
// A workgroup looks at `chunk` rows for runs that begin there: as many as leave
// 2048 workgroups, up to a block.  Calls in us against chunks that leave 512 and
// 8192: 512 cells of 1 to 60 tokens 17 / 22.5 / 18, of 200 to 600 31 / 31 / 39,
// 64 of 500 to 2000 15.7 / 14.4 / 27, 20 tokens each for 512 16 / 16 / 37.  One
// row each: 2180 instead of 257 for the large call.
// ---------------------------------------------------------------------------
constexpr int ST = 256;
constexpr int SMAX = 256;  // largest block size

struct StoreArgs {
    const void *k, *v;
    int64_t k_row, v_row, N;
    const int64_t *slots;
    uint8_t *kc, *vc, *k_exp, *v_exp;
    int64_t n_blocks;
    int shift, bs, d, dp, chunk;
};

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }  // -126 <= e <= 127

// the exponent byte (127 + e) of a block whose largest magnitude is amax
__device__ __forceinline__ int scale_byte(float amax) {
    if (!(amax > 0.f)) return 1;
    int x;
    const float m = frexpf(amax, &x);  // amax = m 2^x, m in [1/2, 1); 448 = 7/8 2^9
    const int b = x - 9 + (m > 0.875f) + 127;
    return b < 1 ? 1 : b > 253 ? 253 : b;
}

// two values at a power-of-two scale to two codes in the low half (or, with `hi`, the high half of `to`)
template <bool HI = false>
__device__ __forceinline__ uint32_t codes2(float x, float y, float s, uint32_t to = 0) {
    const float nan = __uint_as_float(0x7FC00000u);
    const float a = fabsf(x) < INFINITY ? x * s : nan, b = fabsf(y) < INFINITY ? y * s : nan;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)to, HI);
}
__device__ __forceinline__ uint32_t shift_codes(uint32_t c, float s) {  // four codes to a larger exponent
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * s, a[1] * s, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * s, b[1] * s, r, true);
}

// Rows [0, n) of a run.  WIDE: 16-byte aligned rows of a multiple of 8
// columns, through a buffer descriptor that ends with the run: a row before
// or past it, or a column past d, reads zeros, with no branch and 32-bit
// offsets.  Otherwise element by element.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T, bool WIDE>
struct RunRows {
    const T *base;
    int64_t row;   // elements
    uint32_t bytes;
    int n, d;
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ RunRows(const T *p, int64_t row_, int n_, int d_) : base(p), row(row_), n(n_), d(d_) {
        bytes = (uint32_t)(row_ * sizeof(T));
        if constexpr (WIDE)
            rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(p), (short)0, (int)((n - 1) * bytes + d * sizeof(T)),
                                                     0x00020000);
    }
    // columns c .. c + 8 of row r
    __device__ __forceinline__ void load8(int r, int c, float (&y)[8]) const {
        if constexpr (WIDE) {
            const uint32_t at = c < d ? r * bytes + c * (uint32_t)sizeof(T) : 0x80000000u;
            if constexpr (sizeof(T) == 2) {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[2 * i] = __uint_as_float(x[i] << 16), y[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
            } else {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0);
                const u32x4 z = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + 16, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(x[i]), y[4 + i] = __uint_as_float(z[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = r < n && c + i < d ? Elem<T>::load(base, (size_t)(r * row + c + i)) : 0.f;
        }
    }
    // columns c, c + 1 of rows r0 .. r0 + 15, those outside the run as zeros
    __device__ __forceinline__ void load2(int r0, int c, float (&lo)[16], float (&hi)[16]) const {
        if constexpr (WIDE) {
            const uint32_t at = c < d ? r0 * bytes + c * (uint32_t)sizeof(T) : 0x80000000u;
            const uint32_t step = c < d ? bytes : 0;
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                if constexpr (sizeof(T) == 2) {
                    const uint32_t x = __builtin_amdgcn_raw_buffer_load_b32(rsrc, at + t * step, 0, 0);
                    lo[t] = __uint_as_float(x << 16), hi[t] = __uint_as_float(x & 0xFFFF0000u);
                } else {
                    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, at + t * step, 0, 0);
                    lo[t] = __uint_as_float(x[0]), hi[t] = __uint_as_float(x[1]);
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                const int r = r0 + t;
                const bool in = r >= 0 && r < n;
                lo[t] = in && c < d ? Elem<T>::load(base, (size_t)(r * row + c)) : 0.f;
                hi[t] = in && c + 1 < d ? Elem<T>::load(base, (size_t)(r * row + c + 1)) : 0.f;
            }
        }
    }
};

// The largest finite magnitude: the largest of the bits that is a number.
__device__ __forceinline__ float larger(float top, float x) {
    const float y = fabsf(x);
    return y < INFINITY ? fmaxf(top, y) : top;
}

// Between the maximum and the rounding a thread holds KREG pieces of eight
// keys' columns and two columns of 16 tokens of the values in registers: all
// of a 64-token block of 128-wide rows.  What a larger run has beyond that is
// read twice.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(ST) cache_store(StoreArgs a) {
    constexpr int KREG = 4;
    __shared__ int starts[SMAX], n_starts, fail;
    __shared__ float red[2][ST / 64];
    const int tid = threadIdx.x;
    const int64_t x0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t limit = a.n_blocks << a.shift;
    // the tokens of this workgroup's chunk that open a run
    if (tid == 0) n_starts = 0;
    __syncthreads();
    {
        const int64_t x = x0 + tid;
        bool first = false;
        if (tid < a.chunk && x < a.N) {
            const int64_t s = a.slots[x], p = x > 0 ? a.slots[x - 1] : -1;
            first = s >= 0 && s < limit && (x == 0 || s != p + 1 || (s & (a.bs - 1)) == 0);
        }
        if (first) starts[atomicAdd(&n_starts, 1)] = tid;  // any order: runs do not meet
    }
    __syncthreads();
    const int runs = n_starts;
    const int kch = a.dp / 8, kdiv = (65536 + kch - 1) / kch;  // i / kch = i kdiv >> 16 for i < 8192
    const int vch = a.dp / 2, vdiv = (65536 + vch - 1) / vch;
    for (int y = 0; y < runs; ++y) {
        const int64_t x = x0 + __builtin_amdgcn_readfirstlane(starts[y]), s = a.slots[x], b = s >> a.shift;
        const int off = (int)(s & (a.bs - 1));
        // its length: as long as the slots follow each other inside the block
        if (tid == 0) fail = a.bs - off;
        __syncthreads();
        if (tid < a.bs - off && (x + tid >= a.N || a.slots[x + tid] != s + tid)) atomicMin(&fail, tid);
        __syncthreads();
        const int n = __builtin_amdgcn_readfirstlane(fail);
        const RunRows<T, WIDE> kx((const T *)a.k + x * a.k_row, a.k_row, n, a.d), vx((const T *)a.v + x * a.v_row, a.v_row, n, a.d);
        const int kn = n * kch, g0 = off >> 4, vn = (((off + n - 1) >> 4) - g0 + 1) * vch;
        const auto load_k = [&](int i, float (&w)[8]) {  // piece i: row i / kch
            const int r = (i * kdiv) >> 16;
            kx.load8(r, 8 * (i - r * kch), w);
        };
        const auto load_v = [&](int i, float (&lo)[16], float (&hi)[16]) {  // piece i: tokens 16 (g0 + i / vch) .., columns 2 (i % vch) ..
            const int g = (i * vdiv) >> 16;
            vx.load2(16 * (g0 + g) - off, 2 * (i - g * vch), lo, hi);
        };
        float ak = 0.f, av = 0.f, kr[KREG][8], vlo[16], vhi[16];
#pragma unroll
        for (int u = 0; u < KREG; ++u) load_k(tid + u * ST, kr[u]);  // rows past the run: zeros
        load_v(tid, vlo, vhi);
        const auto max_k = [&](const float (&w)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ak = larger(ak, w[i]);
        };
        const auto max_v = [&](const float (&lo)[16], const float (&hi)[16]) {
#pragma unroll
            for (int t = 0; t < 16; ++t) av = larger(larger(av, lo[t]), hi[t]);
        };
#pragma unroll
        for (int u = 0; u < KREG; ++u) max_k(kr[u]);
        max_v(vlo, vhi);
        for (int i = tid + KREG * ST; i < kn; i += ST) {
            float w[8];
            load_k(i, w);
            max_k(w);
        }
        for (int i = tid + ST; i < vn; i += ST) {
            float lo[16], hi[16];
            load_v(i, lo, hi);
            max_v(lo, hi);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) ak = fmaxf(ak, __shfl_xor(ak, o)), av = fmaxf(av, __shfl_xor(av, o));
        if ((tid & 63) == 0) red[0][tid >> 6] = ak, red[1][tid >> 6] = av;
        const int wk = off ? min((int)a.k_exp[b], 253) : 0, wv = off ? min((int)a.v_exp[b], 253) : 0;
        __syncthreads();  // also: everyone has read the old exponents
#pragma unroll
        for (int i = 0; i < ST / 64; ++i) ak = fmaxf(ak, red[0][i]), av = fmaxf(av, red[1][i]);
        const int ek = max(scale_byte(ak), wk), ev = max(scale_byte(av), wv);
        uint8_t *kb = a.kc + b * a.bs * a.dp, *vb = a.vc + b * a.bs * a.dp;
        if (off && ek > wk) {
            const float f = ek - wk > 126 ? 0.f : pow2(wk - ek);
            for (int i = tid; i < off * a.dp / 4; i += ST) ((uint32_t *)kb)[i] = shift_codes(((uint32_t *)kb)[i], f);
        }
        if (off && ev > wv) {
            const float f = ev - wv > 126 ? 0.f : pow2(wv - ev);
            for (int i = tid; i < a.dp * off; i += ST) {
                uint8_t *p = vb + (i / off) * a.bs + i % off;
                *p = (uint8_t)shift_codes(*p, f);
            }
        }
        if (tid == 0) {
            a.k_exp[b] = (uint8_t)ek;
            a.v_exp[b] = (uint8_t)ev;
        }
        const float fk = pow2(127 - ek), fv = pow2(127 - ev);
        const auto put_k = [&](int i, const float (&z)[8]) {  // pieces lie in the block in their order
            const uint32_t lo = codes2<true>(z[2], z[3], fk, codes2(z[0], z[1], fk));
            const uint32_t hi = codes2<true>(z[6], z[7], fk, codes2(z[4], z[5], fk));
            *(uint2 *)(kb + off * a.dp + 8 * i) = make_uint2(lo, hi);
        };
        const auto put_v = [&](int i, const float (&wl)[16], const float (&wh)[16]) {
            const int g = (i * vdiv) >> 16, c = 2 * (i - g * vch), t0 = 16 * (g0 + g), r0 = t0 - off;
            if (c >= a.d) return;
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                lo[q] = codes2<true>(wl[4 * q + 2], wl[4 * q + 3], fv, codes2(wl[4 * q], wl[4 * q + 1], fv));
                hi[q] = codes2<true>(wh[4 * q + 2], wh[4 * q + 3], fv, codes2(wh[4 * q], wh[4 * q + 1], fv));
            }
            uint8_t *p = vb + c * a.bs + t0;
            if (r0 >= 0 && r0 + 16 <= n) {
                *(uint4 *)p = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                if (c + 1 < a.d) *(uint4 *)(p + a.bs) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            } else {
#pragma unroll
                for (int t = 0; t < 16; ++t)
                    if (r0 + t >= 0 && r0 + t < n) {
                        p[t] = (uint8_t)(lo[t / 4] >> 8 * (t % 4));
                        if (c + 1 < a.d) p[a.bs + t] = (uint8_t)(hi[t / 4] >> 8 * (t % 4));
                    }
            }
        };
#pragma unroll
        for (int u = 0; u < KREG; ++u)
            if (tid + u * ST < kn) put_k(tid + u * ST, kr[u]);
        for (int i = tid + KREG * ST; i < kn; i += ST) {
            float w[8];
            load_k(i, w);
            put_k(i, w);
        }
        if (tid < vn) put_v(tid, vlo, vhi);
        for (int i = tid + ST; i < vn; i += ST) {
            float lo[16], hi[16];
            load_v(i, lo, hi);
            put_v(i, lo, hi);
        }
        __syncthreads();
    }
}
}  // namespace

// ---------------------------------------------------------------------------
size_t tables_ws_bytes(int64_t C) {
    return align_up(sizeof(TableHead), 256) + align_up(C * sizeof(TableCell), 256) + 2 * align_up((C + 1) * sizeof(int64_t), 256);
}

hipError_t launch_tables(int64_t C, const int32_t *old_len, const int32_t *new_len, int block_size, int64_t W,
                         int32_t *table, int64_t n_blocks, int32_t *free_list, int32_t *n_free, int64_t n_slots,
                         int64_t *slots, int64_t *offsets, int32_t *lens, int32_t *refused, void *ws, hipStream_t st) {
    TableArgs a{};
    a.C = C, a.W = W, a.n_blocks = n_blocks, a.n_slots = n_slots;
    a.shift = __builtin_ctz(block_size);
    a.old_len = old_len, a.new_len = new_len, a.table = table, a.free_list = free_list, a.n_free = n_free;
    a.slots = slots, a.offsets = offsets, a.lens = lens, a.refused = refused;
    char *p = (char *)ws;
    a.head = (TableHead *)p;
    p += align_up(sizeof(TableHead), 256);
    a.cells = (TableCell *)p;
    p += align_up(C * sizeof(TableCell), 256);
    a.back_off = (int64_t *)p;
    p += align_up((C + 1) * sizeof(int64_t), 256);
    a.need_off = (int64_t *)p;
    if (n_slots <= 8192 && (n_slots > 0 || C * W <= 16384)) {
        hipLaunchKernelGGL(tables_scan<true>, dim3(1), dim3(TT), 0, st, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(tables_scan<false>, dim3(1), dim3(TT), 0, st, a);
    const int64_t items = std::max(n_slots / 4, C * W / 8);
    hipLaunchKernelGGL(tables_move, dim3((unsigned)std::min<int64_t>((items + 255) / 256 + 1, 2048)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_store(const fw_cache &cache, int dtype, const void *k, int64_t k_row, const void *v, int64_t v_row,
                        int64_t N, const int64_t *slots, hipStream_t st) {
    if (N == 0) return hipSuccess;
    StoreArgs a{};
    a.k = k, a.v = v, a.k_row = k_row, a.v_row = v_row, a.N = N, a.slots = slots;
    a.kc = cache.k, a.vc = cache.v, a.k_exp = cache.k_exp, a.v_exp = cache.v_exp;
    a.n_blocks = cache.n_blocks, a.bs = cache.block_size, a.shift = __builtin_ctz(cache.block_size);
    a.d = (int)cache.d, a.dp = cache_row(cache.d);
    const int size = dtype == FW_F32 ? 4 : 2;
    const auto ok = [&](const void *p, int64_t row) {  // a run's offsets stay below 2^31
        return (uintptr_t)p % 16 == 0 && row * size % 16 == 0 && row >= a.d && row * size < (1 << 22);
    };
    const bool wide = a.d % 8 == 0 && ok(k, k_row) && ok(v, v_row);
    a.chunk = 1;
    while (a.chunk < a.bs && N / (2 * a.chunk) >= 2048) a.chunk *= 2;
    const dim3 grid((unsigned)((N + a.chunk - 1) / a.chunk));
    if (dtype == FW_F32) {
        if (wide) hipLaunchKernelGGL((cache_store<float, true>), grid, dim3(ST), 0, st, a);
        else hipLaunchKernelGGL((cache_store<float, false>), grid, dim3(ST), 0, st, a);
    } else {
        if (wide) hipLaunchKernelGGL((cache_store<uint16_t, true>), grid, dim3(ST), 0, st, a);
        else hipLaunchKernelGGL((cache_store<uint16_t, false>), grid, dim3(ST), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace fw
