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
// is served if its running sum of needs stays within top.
//
// tables_scan, one workgroup, takes the sums (each thread a run of cells) and
// writes lengths, offsets and the sums; tables_back and tables_grow, over the
// whole card, move the blocks and write the slots.  Small calls run all three
// in the one workgroup: a launch costs more than their work.
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

// inclusive sums of one value per thread over the workgroup; `red` holds TT / 64 values
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *red, int64_t *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t y = __shfl_up(v, off);
        if (lane >= off) v += y;
    }
    if (lane == 63) red[w] = v;
    __syncthreads();
    int64_t before = 0, sum = 0;
    for (int i = 0; i < TT / 64; ++i) {
        if (i < w) before += red[i];
        sum += red[i];
    }
    __syncthreads();
    *total = sum;
    return v + before;
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

// slots of tokens i .. i + 3; new blocks straight off the stack (take_blocks writes the same into the table)
__device__ __forceinline__ void write_slots(const TableArgs &a, const TableHead &hd, int64_t n, int64_t first, int64_t step) {
    const int64_t mask = ((int64_t)1 << a.shift) - 1;
    for (int64_t i0 = 4 * first; i0 < n; i0 += 4 * step) {
        int64_t c = find_cell(a.offsets, a.C, i0);
        for (int64_t i = i0; i < i0 + 4 && i < n; ++i) {
            while (i >= a.offsets[c + 1]) ++c;
            const TableCell t = a.cells[c];
            const int64_t pos = t.old_len + (i - a.offsets[c]), b = pos >> a.shift;
            int64_t s = -1;
            if (t.served) {
                const int32_t e = b < t.had ? a.table[c * a.W + b] : a.free_list[hd.top - 1 - (a.need_off[c] + b - t.had)];
                if (e >= 0) s = ((int64_t)e << a.shift) + (pos & mask);
            }
            a.slots[i] = s;
        }
    }
}

__device__ __forceinline__ int64_t slot_count(const TableArgs &a) {
    const int64_t n = a.offsets[a.C];
    return a.slots ? (n < a.n_slots ? n : a.n_slots) : 0;
}

template <bool ALL>
__global__ void __launch_bounds__(TT) tables_scan(TableArgs a) {
    __shared__ int64_t red[TT / 64];
    const int64_t run = (a.C + TT - 1) / TT, c0 = threadIdx.x * run;
    const int64_t c1 = c0 + run < a.C ? c0 + run : a.C;
    int64_t back = 0, need = 0, add = 0;
    for (int64_t c = c0; c < c1; ++c) {
        const CellPlan p = plan_cell(a, c);
        back += p.back, need += p.need, add += p.add;
    }
    int64_t n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : n_free > a.n_blocks ? a.n_blocks : n_free;
    TableHead hd;
    int64_t total;
    int64_t ob = block_scan(back, red, &hd.back) - back;
    int64_t on = block_scan(need, red, &total) - need;
    if (threadIdx.x == TT - 1) a.need_off[a.C] = total;
    int64_t oa = block_scan(add, red, &total) - add;
    if (threadIdx.x == TT - 1) a.offsets[a.C] = total, a.back_off[a.C] = hd.back;
    hd.n_free = n_free;
    hd.top = n_free + hd.back < a.n_blocks ? n_free + hd.back : a.n_blocks;
    int64_t take = 0, refused = 0;
    for (int64_t c = c0; c < c1; ++c) {
        const CellPlan p = plan_cell(a, c);
        const bool served = p.fits && on + p.need <= hd.top;
        a.cells[c] = TableCell{p.o, (int32_t)p.had, (int32_t)p.want, served};
        a.back_off[c] = ob, a.need_off[c] = on, a.offsets[c] = oa;
        if (served) take = on + p.need;
        refused += !served;
        a.lens[c] = served ? p.n : p.o;   // may be old_len: this thread alone reads and writes the cell
        ob += p.back, on += p.need, oa += p.add;
    }
    // running sums only grow, so what is taken is the largest served one
    block_scan(refused, red, &total);
    if (threadIdx.x == 0) a.refused[0] = (int32_t)total;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int64_t y = __shfl_xor(take, off);
        take = y > take ? y : take;
    }
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = take;
    __syncthreads();
    for (int i = 0; i < TT / 64; ++i) take = red[i] > take ? red[i] : take;
    hd.take = take;
    if (threadIdx.x == 0) {
        a.head[0] = hd;
        a.n_free[0] = (int32_t)(hd.top - hd.take);
    }
    if (ALL) {
        __syncthreads();  // the cells' records are read by every thread from here on
        move_back(a, hd, threadIdx.x, TT);
        __syncthreads();  // blocks that just came back may be taken
        take_blocks(a, hd, threadIdx.x, TT);
        write_slots(a, hd, slot_count(a), threadIdx.x, TT);
    }
}

__global__ void __launch_bounds__(256) tables_back(TableArgs a) {
    move_back(a, a.head[0], (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

__global__ void __launch_bounds__(256) tables_grow(TableArgs a) {
    const TableHead hd = a.head[0];
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    take_blocks(a, hd, first, step);
    write_slots(a, hd, slot_count(a), first, step);
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

__device__ __forceinline__ float finite_abs(float x) {
    x = fabsf(x);
    return x < INFINITY ? x : 0.f;
}

// two values at a power-of-two scale to two codes in the low half
__device__ __forceinline__ uint32_t codes2(float x, float y, float s) {
    const float nan = __uint_as_float(0x7FC00000u);
    const float a = fabsf(x) < INFINITY ? x * s : nan, b = fabsf(y) < INFINITY ? y * s : nan;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}
__device__ __forceinline__ uint32_t shift_codes(uint32_t c, float s) {  // four codes to a larger exponent
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * s, a[1] * s, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * s, b[1] * s, r, true);
}

template <typename T>
__global__ void __launch_bounds__(ST) cache_store(StoreArgs a) {
    __shared__ int starts[SMAX], n_starts, fail;
    __shared__ float red[ST / 64];
    const int64_t x0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t limit = a.n_blocks << a.shift;
    const T *k = (const T *)a.k, *v = (const T *)a.v;
    // the tokens of this workgroup's chunk that open a run
    if (threadIdx.x == 0) n_starts = 0;
    __syncthreads();
    {
        const int64_t x = x0 + threadIdx.x;
        bool first = false;
        if ((int)threadIdx.x < a.chunk && x < a.N) {
            const int64_t s = a.slots[x], p = x > 0 ? a.slots[x - 1] : -1;
            first = s >= 0 && s < limit && (x == 0 || s != p + 1 || (s & (a.bs - 1)) == 0);
        }
        if (first) starts[atomicAdd(&n_starts, 1)] = threadIdx.x;  // any order: runs do not meet
    }
    __syncthreads();
    const int runs = n_starts;
    for (int y = 0; y < runs; ++y) {
        const int64_t x = x0 + starts[y], s = a.slots[x], b = s >> a.shift;
        const int off = (int)(s & (a.bs - 1));
        // its length: as long as the slots follow each other inside the block
        if (threadIdx.x == 0) fail = a.bs - off;
        __syncthreads();
        if ((int)threadIdx.x < a.bs - off && (x + threadIdx.x >= a.N || a.slots[x + threadIdx.x] != s + threadIdx.x))
            atomicMin(&fail, (int)threadIdx.x);
        __syncthreads();
        const int n = fail;
        float ak = 0.f, av = 0.f;
        for (int i = threadIdx.x; i < n * a.d; i += ST) {
            const int r = i / a.d, c = i % a.d;
            ak = fmaxf(ak, finite_abs(Elem<T>::load(k, (size_t)((x + r) * a.k_row + c))));
            av = fmaxf(av, finite_abs(Elem<T>::load(v, (size_t)((x + r) * a.v_row + c))));
        }
        ak = block_reduce(ak, red, OpMax());
        av = block_reduce(av, red, OpMax());
        const int wk = off ? min((int)a.k_exp[b], 253) : 0, wv = off ? min((int)a.v_exp[b], 253) : 0;
        const int ek = max(scale_byte(ak), wk), ev = max(scale_byte(av), wv);
        uint8_t *kb = a.kc + b * a.bs * a.dp, *vb = a.vc + b * a.bs * a.dp;
        if (off && ek > wk) {
            const float f = ek - wk > 126 ? 0.f : pow2(wk - ek);
            for (int i = threadIdx.x; i < off * a.dp / 4; i += ST) ((uint32_t *)kb)[i] = shift_codes(((uint32_t *)kb)[i], f);
        }
        if (off && ev > wv) {
            const float f = ev - wv > 126 ? 0.f : pow2(wv - ev);
            for (int i = threadIdx.x; i < a.dp * off; i += ST) {
                uint8_t *p = vb + (i / off) * a.bs + i % off;
                *p = (uint8_t)shift_codes(*p, f);
            }
        }
        __syncthreads();  // everyone has read the old exponents
        if (threadIdx.x == 0) {
            a.k_exp[b] = (uint8_t)ek;
            a.v_exp[b] = (uint8_t)ev;
        }
        const float fk = pow2(127 - ek), fv = pow2(127 - ev);
        for (int i = threadIdx.x; i < n * a.dp / 2; i += ST) {
            const int r = i / (a.dp / 2), c = 2 * (i % (a.dp / 2));
            const float p = c < a.d ? Elem<T>::load(k, (size_t)((x + r) * a.k_row + c)) : 0.f;
            const float q = c + 1 < a.d ? Elem<T>::load(k, (size_t)((x + r) * a.k_row + c + 1)) : 0.f;
            *(uint16_t *)(kb + (off + r) * a.dp + c) = (uint16_t)codes2(p, q, fk);
        }
        for (int i = threadIdx.x; i < n * a.d; i += ST) {
            const int r = i / a.d, c = i % a.d;
            vb[c * a.bs + off + r] = (uint8_t)codes2(Elem<T>::load(v, (size_t)((x + r) * a.v_row + c)), 0.f, fv);
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
    if ((n_slots > 0 && n_slots <= 8192) || C * W <= 16384) {
        hipLaunchKernelGGL(tables_scan<true>, dim3(1), dim3(TT), 0, st, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(tables_scan<false>, dim3(1), dim3(TT), 0, st, a);
    const auto blocks = [](int64_t items) { return (unsigned)std::min<int64_t>(std::max<int64_t>((items + 255) / 256, 1), 2048); };
    hipLaunchKernelGGL(tables_back, dim3(blocks(C * W / 8)), dim3(256), 0, st, a);
    hipLaunchKernelGGL(tables_grow, dim3(blocks(std::max(n_slots / 4, C * W / 8))), dim3(256), 0, st, a);
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
    a.chunk = 1;
    while (a.chunk < a.bs && N / (2 * a.chunk) >= 2048) a.chunk *= 2;
    const dim3 grid((unsigned)((N + a.chunk - 1) / a.chunk));
    if (dtype == FW_F32) hipLaunchKernelGGL(cache_store<float>, grid, dim3(ST), 0, st, a);
    else hipLaunchKernelGGL(cache_store<uint16_t>, grid, dim3(ST), 0, st, a);
    return hipGetLastError();
}

}  // namespace fw
