// Cells that share blocks of the 8-bit cache: fw_cache_fork, fw_cache_release
// and fw_cache_compact.
//
// shared[b] counts the cells that hold block b besides its first.  A cell that
// leaves a block takes one off; who finds none was the last, and sets the
// block's bit.  The marked blocks go on the stack in ascending order, so the
// result does not depend on who came last: collect_blocks finds their places by
// counting bits.  Blocks that a call takes come from the stack as it was
// before, so no block that others hold is written.
//
// What bounds them: a fork of 2048 cells from 256 cells of 3000 to 30000 tokens,
// after they were ended, takes 51 us: 7 and 9 in which one workgroup serves the
// requests in order (a chain of loads), 14 for the counters of 300000
// blocks down, 4 for the stack, 17 for them up and 2048 part-filled blocks (67
// MB, 13 at the rate of a copy).  A counter for each run of blocks instead of the
// bits took 480: atomics at one address come one by one, 10 ns each.  The one
// workgroup's time grows with the requests: 40 us for 7936 forks (the copies 33
// beside it), 400 for 65280 (357); 570 for a release that looks at 65536 cells and
// cuts none.
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int PT = 1024;    // threads of the one workgroup that serves cells in order
constexpr int WT = 256;     // threads of the others
constexpr int kRun = 16 * WT;  // blocks that one workgroup puts back

struct PageHead {
    int64_t top, left;  // free blocks before the call, and without those it takes
};

struct PageArgs {
    int64_t C, W, n_blocks, P, n_kept, nruns, chunks;
    int shift, bs, polls, dp;
    int32_t *table, *lens, *free_list, *n_free, *shared, *refused;
    uint8_t *kc, *vc, *k_exp, *v_exp;
    const int32_t *new_len, *src, *dst, *length, *which, *kept_pos;
    const int64_t *offsets;
    // workspace
    PageHead *head;
    uint16_t *marks;      // [nruns][WT] a bit for each block that its last cell left
    int32_t *counts;      // [nruns] how many, where runs are many
    int32_t *claim;       // [C] the first pair or listed cell that names a cell
    int4 *plan;           // [max(C, P)] per cell, pair or listed cell
    // compaction
    int32_t *rank;        // [blocks kept] rank among the blocks that the cell takes, or -1
    int32_t *taken;       // [blocks kept] the blocks taken, in their order
    int32_t *owner;       // [chunks] listed cell, or -1
    int32_t *within;      // [chunks] of the cell's kept tokens, the first that lies in or behind the chunk's own positions
    int32_t *read;        // [2][chunks] set once the chunk's keys, and values, have been read
    int32_t *tickets;     // [2 kQueues][kApart] chunks handed out, of keys and of values
    int32_t *starts;      // [kQueues + 1] first chunk of each queue; all equal if nothing moves
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
    if (!is_block(a, b)) return;
    if (atomicSub(&a.shared[b], 1) > 0) return;
    __hip_atomic_store(&a.shared[b], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    atomicOr((uint32_t *)a.marks + (b >> 5), 1u << (b & 31));
}

// A block's codes and exponents, by a workgroup of WT threads.
__device__ __forceinline__ void copy_block(const PageArgs &a, int32_t from, int32_t to) {
    const int64_t n = (int64_t)a.bs * a.dp;
    const uint4 *k0 = (const uint4 *)(a.kc + from * n), *v0 = (const uint4 *)(a.vc + from * n);
    uint4 *k1 = (uint4 *)(a.kc + to * n), *v1 = (uint4 *)(a.vc + to * n);
#pragma unroll 2
    for (int i = threadIdx.x; i < n / 16; i += WT) {
        const uint4 x = k0[i], y = v0[i];
        k1[i] = x, v1[i] = y;
    }
    if (threadIdx.x == 0) a.k_exp[to] = a.k_exp[from], a.v_exp[to] = a.v_exp[from];
}

// Serves `n` requests in order, each thread a run of them: need(i) blocks (0 or more) for request i, -1 for one that is
// refused in any case.  done(i, served, first): its first block's rank among those taken.  Counts those refused, and
// leaves the stack's heights in the head.  A run of up to kAsk is asked for once, a longer one twice (the fork above
// 2 us less than with two askings).
constexpr int kAsk = 4;
template <typename Need, typename Done>
__device__ __forceinline__ void serve(const PageArgs &a, int64_t n, const Need &need, const Done &done) {
    __shared__ int64_t red[PT / 64];
    __shared__ int32_t refused;
    __shared__ unsigned long long taken;
    if (threadIdx.x == 0) refused = 0, taken = 0;
    const int64_t run = (n + PT - 1) / PT, i0 = threadIdx.x * run, i1 = i0 + run < n ? i0 + run : n;
    int64_t mine = 0, all, ask[kAsk];
    const int64_t top = free_blocks(a);
    if (run <= kAsk) {
#pragma unroll
        for (int u = 0; u < kAsk; ++u) {
            ask[u] = i0 + u < i1 ? need(i0 + u) : 0;
            mine += ask[u] > 0 ? ask[u] : 0;
        }
    } else {
        for (int64_t i = i0; i < i1; ++i) {
            const int64_t x = need(i);
            mine += x > 0 ? x : 0;
        }
    }
    int64_t at = sum_before<PT>(mine, red, &all);
    int64_t last = 0;
    int32_t out = 0;
    const auto one = [&](int64_t i, int64_t x) {
        const int64_t want = x > 0 ? x : 0;
        const bool served = x == 0 || (x > 0 && at + x <= top);
        if (served && want) last = at + want;
        out += !served;
        done(i, served, x, at);
        at += want;
    };
    if (run <= kAsk) {
#pragma unroll
        for (int u = 0; u < kAsk; ++u)
            if (i0 + u < i1) one(i0 + u, ask[u]);
    } else {
        for (int64_t i = i0; i < i1; ++i) one(i, need(i));
    }
    if (out) atomicAdd(&refused, out);
    // running sums only grow: a wave's last one is its highest lane's
    const uint64_t any = __ballot(last > 0);
    if (any) {
        const int hi = 63 - __builtin_clzll(any);
        if ((int)(threadIdx.x & 63) == hi) atomicMax(&taken, (unsigned long long)last);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        a.refused[0] = refused;
        a.head[0] = PageHead{top, top - (int64_t)taken};
    }
}
__device__ __forceinline__ int32_t fresh_block(const PageArgs &a, int64_t top, int64_t rank) { return a.free_list[top - 1 - rank]; }

// by workgroup b of nb
__device__ __forceinline__ void clear_marks(const PageArgs &a, int64_t b, int64_t nb) {
    for (int64_t i = b * blockDim.x + threadIdx.x; i < a.nruns * (WT / 4); i += nb * blockDim.x) ((uint64_t *)a.marks)[i] = 0;
}

// Runs up to which collect_blocks counts the marks of those before its own from their bits; many have their numbers
// counted first, and marks that many workgroups clear (a release of nothing among 260000 blocks, 64 runs: 19 us, with the
// two launches 25; among 1000000, 245 runs: 25 either way).
constexpr int64_t kFewRuns = 64;

__global__ void __launch_bounds__(WT) clear_all(PageArgs a) { clear_marks(a, blockIdx.x, gridDim.x); }

__global__ void __launch_bounds__(WT) count_runs(PageArgs a) {
    __shared__ int64_t red[WT / 64];
    int64_t all;
    sum_before<WT>(__popc(a.marks[(int64_t)blockIdx.x * WT + threadIdx.x]), red, &all);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = (int32_t)all;
}

// A run's marked blocks onto the stack, by a workgroup.
__device__ __forceinline__ void collect_run(const PageArgs &a, int64_t run) {
    __shared__ int64_t red[WT / 64];
    int64_t before = 0, upto, here;
    if (a.nruns <= kFewRuns)
        for (int64_t i = threadIdx.x; i < run * (WT / 4); i += WT) before += __popcll(((const uint64_t *)a.marks)[i]);
    else
        for (int64_t i = threadIdx.x; i < run; i += WT) before += a.counts[i];
    uint32_t m = a.marks[run * WT + threadIdx.x];
    sum_before<WT>(before, red, &upto);
    int64_t at = a.head[0].left + upto + sum_before<WT>(__popc(m), red, &here);
    if (run == a.nruns - 1 && threadIdx.x == 0) {
        const int64_t n = a.head[0].left + upto + here;
        a.n_free[0] = (int32_t)(n < a.n_blocks ? n : a.n_blocks);
    }
    const int64_t b0 = 16 * (run * WT + threadIdx.x);
    for (; m; m &= m - 1, ++at)
        if (at < a.n_blocks) a.free_list[at] = (int32_t)(b0 + __builtin_ctz(m));
}
__global__ void __launch_bounds__(WT) collect_blocks(PageArgs a) { collect_run(a, blockIdx.x); }

// ---------------------------------------------------------------------------
// release: plan = (blocks kept, blocks held, block for the copy or -1, served)
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(PT) release_plan(PageArgs a) {
    if (a.nruns <= kFewRuns) clear_marks(a, 0, 1);
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
    serve(a, a.C, need, [&](int64_t c, bool served, int64_t x, int64_t first) {
        int64_t old;
        const int64_t n = cut(c, &old);
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
// Who is the first of `n` to name a cell (claims in LDS measured the same at 2048 cells).
__device__ __forceinline__ int32_t claimed(const PageArgs &a, int32_t c) {
    return __hip_atomic_load(&a.claim[c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void claim_cells(const PageArgs &a, int64_t n, const int32_t *cells) {
    for (int64_t p = threadIdx.x; p < n; p += PT)
        if (in_range(a, cells[p])) __hip_atomic_store(&a.claim[cells[p]], INT32_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int64_t p = threadIdx.x; p < n; p += PT)
        if (in_range(a, cells[p])) atomicMin(&a.claim[cells[p]], (int32_t)p);
    __syncthreads();
}

__global__ void __launch_bounds__(PT) fork_plan(PageArgs a) {
    const auto tokens = [&](int64_t p) -> int64_t {  // of pair p, or -1; whether it is the first to name its cell aside
        const int32_t s = a.src[p], t = a.dst[p];
        const bool ok = in_range(a, s) && in_range(a, t);
        const int64_t n = length_of(a, ok ? s : 0), is = length_of(a, ok ? t : 0), most = a.length ? a.length[p] : n;
        return !ok || is != 0 ? -1 : most >= n ? n : most > 0 ? most : 0;
    };
    const auto if_first = [&](int64_t p, int64_t n) { return n >= 0 && claimed(a, a.dst[p]) == p ? n : -1; };
    const auto blocks = [&](int64_t n) -> int64_t { return n < 0 ? -1 : (n & (a.bs - 1)) != 0; };
    const int64_t top = free_blocks(a);
    const auto done = [&](int64_t p, bool served, int64_t x, int64_t first, int64_t n) {
        a.plan[p] = make_int4(served ? (int)n : -1, served && x ? fresh_block(a, top, first) : -1, 0, 0);
        if (served) a.lens[a.dst[p]] = (int)n;
    };
    // lengths of before the call: all are read before any is written
    const int64_t run = (a.P + PT - 1) / PT, i0 = threadIdx.x * run;
    if (run <= kAsk) {
        int64_t n[kAsk];
#pragma unroll
        for (int u = 0; u < kAsk; ++u) n[u] = u < run && i0 + u < a.P ? tokens(i0 + u) : -1;
        claim_cells(a, a.P, a.dst);
        serve(a, a.P, [&](int64_t p) { return blocks(n[p - i0] = if_first(p, n[p - i0])); },
              [&](int64_t p, bool served, int64_t x, int64_t first) { done(p, served, x, first, n[p - i0]); });
    } else {
        claim_cells(a, a.P, a.dst);
        for (int64_t p = threadIdx.x; p < a.P; p += PT) a.plan[p].x = (int)if_first(p, tokens(p));
        __syncthreads();
        serve(a, a.P, [&](int64_t p) { return blocks(a.plan[p].x); },
              [&](int64_t p, bool served, int64_t x, int64_t first) { done(p, served, x, first, a.plan[p].x); });
    }
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
// The tokens that a listed cell keeps fall into chunks of kChunk, one or more
// blocks each.  Chunk j of listed cell p is number offsets[p] / kChunk + p + j
// (and block j number offsets[p] / bs + p + j): ascending offsets leave room for
// every cell's chunks, so none needs to be counted before.
// plan = (tokens kept or -1, first block that changes, blocks to take, first of them)
//
// Tokens move inside their cell's own blocks, towards the front, so a chunk's
// blocks may be written once the chunks that keep tokens of them, none of them
// behind the chunk itself, have read theirs.  compact_move's workgroups take
// chunks, keys and values apart, by ticket: they read all they need into LDS,
// say so, wait for the chunks before theirs that read their blocks, and write.
// Tickets come from queues of whole cells, each in the order of its chunks, and
// a workgroup takes its next one before it is done with the one at hand.  So a
// chunk waits for chunks of earlier tickets of its queue, and is waited for at
// most until its workgroup is done with that of its ticket before: always for
// what was handed out earlier, so every wait ends.
//
// Memory bounds it: 256 cells of 6000 to 60000 tokens of 128 columns of which
// 0.3 stay, 443 MB of kept tokens, for which 700 MB are read and written in whole
// lines (values lie tokens innermost), take 193 us in compact_move (4 TB/s of
// what its counters see), 227 in all.  Two passes through buffers of their own
// took 273 for the reads alone.  Keys and values in launches of their own: 275 in
// all.  One queue for all: 26000 tickets at one address, 10 ns each.
// ---------------------------------------------------------------------------
constexpr int CT = 1024;     // threads that look through a cell's list
constexpr int MT = 512;      // threads that move a chunk
constexpr int kMovers = 768;  // workgroups of it, three to a compute unit (the size above: 247 us, two 254, four 264)
constexpr int kChunk = 256;  // tokens
constexpr int kChunkShift = 8;
constexpr int kQueues = 64;  // of keys, and as many of values
constexpr int kApart = 64;   // counters lie in lines of their own
// Looks at flags before a wait is given up, seconds: a wait ends also if another call overwrites the workspace, which
// no caller may do.  The chunk is then left unwritten and `refused` becomes -1.
constexpr int kPolls = 1 << 22;

__device__ __forceinline__ int64_t cell_of(const PageArgs &a, int64_t p) { return a.which ? a.which[p] : p; }
__device__ __forceinline__ int64_t block0(const PageArgs &a, int64_t p) { return (a.offsets[p] >> a.shift) + p; }
__device__ __forceinline__ int64_t chunk0(const PageArgs &a, int64_t p) { return (a.offsets[p] >> kChunkShift) + p; }
// offsets of refused cells can be anything
__device__ __forceinline__ int64_t clamp_chunk(const PageArgs &a, int64_t t) { return t < 0 ? 0 : t > a.chunks ? a.chunks : t; }

__global__ void __launch_bounds__(CT) compact_check(PageArgs a) {
    __shared__ int64_t red[CT / 64];
    const int64_t p = blockIdx.x, c = cell_of(a, p);
    const int64_t o = a.offsets[p], e = a.offsets[p + 1], n = e - o;
    const int tid = threadIdx.x;
    clear_marks(a, p, a.P);
    for (int64_t i = p * CT + tid; i < 2 * a.chunks; i += a.P * CT) a.read[i] = 0;
    if (p == 0 && tid < 2 * kQueues) a.tickets[tid * kApart] = 0;
    bool bad = c < 0 || c >= a.C || o < 0 || e > a.n_kept || n < 0;
    const int64_t len = bad ? 0 : length_of(a, c);
    bad = bad || n > len;
    // chunks of no cell before the first, behind this one's, and behind the last
    const int64_t t0 = chunk0(a, p), t1 = bad ? t0 : t0 + ((n + kChunk - 1) >> kChunkShift);
    const int64_t next = p + 1 < a.P ? chunk0(a, p + 1) : a.chunks;
    if (p == 0)
        for (int64_t t = tid; t < clamp_chunk(a, t0); t += CT) a.owner[t] = -1;
    for (int64_t t = clamp_chunk(a, t0) + tid; t < clamp_chunk(a, next); t += CT) a.owner[t] = t < t1 ? (int32_t)p : -1;
    // the first blocks' owners, beside the list
    const int32_t *row = a.table + c * a.W;
    bool early = false;
    if (!bad && tid < nb(a, n)) {
        const int32_t b = row[tid];
        early = is_block(a, b) && a.shared[b] > 0;
    }
    int64_t stay = 0;
    if (!bad) {
        const int32_t *pos = a.kept_pos + o;
        const int64_t last = ((n + kChunk - 1) >> kChunkShift) - 1;
        int32_t ahead[5];  // positions i0 - 1 .. i0 + 3, a step ahead
        const auto load = [&](int64_t i0) {
#pragma unroll
            for (int u = 0; u < 5; ++u) ahead[u] = i0 + u == 0 ? -1 : pos[i0 + u - 1 < n ? i0 + u - 1 : n - 1];
        };
        if (4 * tid < n) load(4 * tid);
        for (int64_t i0 = 4 * tid; i0 < n; i0 += 4 * CT) {
            int64_t z[5];
#pragma unroll
            for (int u = 0; u < 5; ++u) z[u] = ahead[u];
            if (i0 + 4 * CT < n) load(i0 + 4 * CT);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t i = i0 + u, x = z[u + 1], y = z[u];
                if (i >= n) break;
                bad = bad || x <= y || x >= len || x < i;
                if (bad) break;
                stay += x == i;
                // chunks of positions that begin behind the token before and not behind this one
                for (int64_t b = y < 0 ? 0 : (y >> kChunkShift) + 1; b <= x >> kChunkShift && b <= last; ++b)
                    a.within[t0 + b] = (int32_t)i;
            }
        }
    }
    bad = __syncthreads_or(bad);
    if (bad) {
        if (tid == 0) a.plan[p] = make_int4(-1, 0, 0, 0);
        return;
    }
    int64_t fixed;
    sum_before<CT>(stay, red, &fixed);  // positions ascend: the tokens that stay come first
    int64_t first = fixed >> a.shift;
    if (fixed == n && (n & (a.bs - 1))) {
        const int32_t b = row[first];
        if (!is_block(a, b) || a.shared[b] <= 0) ++first;
    }
    int64_t take = 0;
    const int64_t b0 = block0(a, p);
    for (int64_t j0 = 0; j0 < nb(a, n); j0 += CT) {
        const int64_t j = j0 + tid;
        bool other = early;
        if (j0 > 0) {
            const int32_t b = j < nb(a, n) ? row[j] : -1;
            other = is_block(a, b) && a.shared[b] > 0;
        }
        other = other && j >= first;
        int64_t all;
        const int64_t before = sum_before<CT>(other, red, &all);
        if (j < nb(a, n)) a.rank[b0 + j] = other ? (int32_t)(take + before) : -1;
        take += all;
    }
    if (tid == 0) a.plan[p] = make_int4((int)n, (int)first, (int)take, 0);
}

__global__ void __launch_bounds__(PT) compact_plan(PageArgs a) {
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
          [&](int64_t p, bool served, int64_t, int64_t first) {
              if (!served) a.plan[p].x = -1;
              else a.plan[p].w = (int)first;
          });
    // queue i begins with the first cell whose chunks begin at i / kQueues of all or behind; the first with chunk 0
    if (down && threadIdx.x <= kQueues) a.starts[threadIdx.x] = 0;
    for (int64_t p = threadIdx.x; p <= a.P && !down; p += PT) {
        const int64_t t = p < a.P ? clamp_chunk(a, chunk0(a, p)) : a.chunks;
        const int64_t before = p > 0 ? clamp_chunk(a, chunk0(a, p - 1)) : -1;
        for (int64_t i = before < 0 ? 0 : before * kQueues / a.chunks; i <= kQueues; ++i) {
            const int64_t at = i * a.chunks / kQueues;
            if (at > t) break;
            if (at > before) a.starts[i] = i == 0 ? 0 : (int32_t)t;
        }
    }
}

// A code's magnitude in an order with 0 below 1, NaN below all (four bytes at a time).
__device__ __forceinline__ uint32_t magnitudes(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x7F7F7F7Fu; }
// The least exponent byte for a magnitude (as above) at exponent byte e; 0 for zero.
__device__ __forceinline__ int least_exp(int magnitude, int e) {
    if (magnitude < 2) return 0;
    const float v = __builtin_amdgcn_cvt_pk_f32_fp8(magnitude - 1, false)[0];
    int x;
    const float m = frexpf(v, &x);  // 448 = 7/8 2^9
    return x - 9 + (m > 0.875f) + e;
}
__device__ __forceinline__ float exp_ratio(int from, int to) {  // 2^(from - to): codes that are not 0 stay in range
    const int e = from - to;
    return __uint_as_float((uint32_t)(127 + (e < -126 ? -126 : e > 127 ? 127 : e)) << 23);
}
__device__ __forceinline__ uint32_t scale_codes(uint32_t c, float s0, float s1, float s2, float s3) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * s0, a[1] * s1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * s2, b[1] * s3, r, true);
}
__device__ __forceinline__ int exp_byte(uint8_t e) { return e < 1 ? 1 : e > 253 ? 253 : e; }
__device__ __forceinline__ uint32_t max_bytes(uint32_t x, uint32_t y) {  // bytes below 0x80
    const uint32_t more = ((x | 0x80808080u) - y) & 0x80808080u;          // where x >= y
    const uint32_t keep = more - (more >> 7) | more;
    return (x & keep) | (y & ~keep);
}

// LDS: a chunk's codes, keys [token][dp] or values [dp][kChunk + 4] (the padding spreads a column over the banks).
//
// Values lie tokens innermost, so whole blocks are read for the tokens that
// stay.  A load takes 16 tokens of a row in each lane, neighbouring lanes
// neighbouring bytes (a line of memory that a second load asks for while it is
// still on its way holds up the compute unit's cache), and a lane packs the
// bytes that stay: byte permutes whose selectors a table has for every choice of
// a word's bytes and every place in the output word.  Words that two lanes fill
// together are joined by LDS atomics, each byte written once.
struct MoveShared {
    alignas(16) uint64_t stay[kChunk];  // values: tokens of the group that stay; then the tokens' ratios and magnitudes
    uint2 pack[64];        // selectors for four bits of these and 0 .. 3 bytes that are there
    int2 place[kChunk];
    int32_t blk[kChunk];   // keys: a token's block; values: the block of a group of up to 64 neighbours
    int32_t info[kChunk];  // keys: its place there; values: the group's first token, and 8 its place
    int16_t ex[kChunk];
    int32_t to[kChunk / 16];
    int least[kChunk / 16];
    int32_t ticket, count[kChunk / 64];
};

template <bool VALUES, bool ONCE>
__device__ __forceinline__ void move_chunks(const PageArgs &a, uint8_t *const lds, MoveShared &sh) {
    auto &stay = sh.stay;
    auto &pack = sh.pack;
    auto &place = sh.place;
    auto &blk = sh.blk, &info = sh.info;
    auto &to = sh.to;
    auto &ex = sh.ex;
    auto &least = sh.least;
    auto &s_count = sh.count;
    int32_t &s_ticket = sh.ticket;
    float *const ratio = (float *)stay;  // once the tokens are packed
    uint32_t *const top = (uint32_t *)stay + kChunk;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t size = (int64_t)a.bs * a.dp;
    constexpr int vrow = kChunk + 4;
    // The last wave takes the tickets, a lane for each queue: the next one while the chunk at hand is waited for.
    int32_t *const tickets = a.tickets + VALUES * kQueues * kApart, *const read = a.read + VALUES * a.chunks;
    const int q_first = a.starts[lane], q_size = a.starts[lane + 1] - q_first;
    uint64_t open = __ballot(q_size > 0);  // queues that may have tickets left
    const auto take_ticket = [&]() {
        int32_t got = -1;
        while (open) {
            const int from = blockIdx.x & 63;
            const int q = (__builtin_ctzll(open >> from | open << (64 - from & 63)) + from) & 63;
            int32_t n = 0;
            if (lane == q) n = atomicAdd(&tickets[lane * kApart], 1);
            n = __builtin_amdgcn_readlane(n, q);
            if (n < __builtin_amdgcn_readlane(q_size, q)) {
                got = __builtin_amdgcn_readlane(q_first, q) + n;
                break;
            }
            // a look at all of them, only now: everyone reads the same few lines
            open &= __ballot(__hip_atomic_load(&tickets[lane * kApart], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < q_size);
        }
        if (lane == 0) s_ticket = got;
    };
    __syncthreads();
    if (VALUES && tid < 64) {
        const int fill = tid & 3;
        int k = 0;
        uint32_t bytes = 0, join = 0, rest = 0;
        for (int i = 0; i < 4; ++i)
            if (tid >> (2 + i) & 1) bytes |= (uint32_t)i << (8 * k++);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // bytes 4 .. 7 are the output word's, 0 .. 3 the new ones, 0x0c is zero
            const int on = i - fill, up = i + 4 - fill;
            join |= (i < fill ? 4u + i : on < k ? (bytes >> (8 * on)) & 0xFFu : 0x0Cu) << (8 * i);
            rest |= (up < k ? (bytes >> (8 * up)) & 0xFFu : 0x0Cu) << (8 * i);
        }
        pack[tid] = make_uint2(join, rest);
    }
    if (w == MT / 64 - 1) take_ticket();
    for (;;) {
    __syncthreads();  // the ticket is there, and what the chunk before left in LDS is done with
    const int32_t chunk = __builtin_amdgcn_readfirstlane(s_ticket);
    if (chunk < 0) return;
    const int32_t p = a.owner[chunk];
    const int4 x = p < 0 ? make_int4(-1, 0, 0, 0) : a.plan[p];
    const int64_t o = p < 0 ? 0 : a.offsets[p], t0 = (o >> kChunkShift) + p, j = chunk - t0;
    // this chunk's tokens in blocks that change
    const int lo = (int)max((int64_t)x.y * a.bs - j * kChunk, (int64_t)0), hi = (int)min(x.x - j * kChunk, (int64_t)kChunk);
    if (ONCE) open = 0;
    if (p < 0 || lo >= hi) {
        __syncthreads();  // everyone has the ticket
        if (w == MT / 64 - 1) take_ticket();
        continue;
    }
    if (tid < kChunk / 16) least[tid] = 1;
    const int32_t *row = a.table + cell_of(a, p) * a.W;
    const uint8_t *codes = VALUES ? a.vc : a.kc, *exps = VALUES ? a.v_exp : a.k_exp;
    // where each token lies
    const bool mine = tid >= lo && tid < hi;
    int b = -1, off = 0, e = 1;
    if (mine) {
        const int y = a.kept_pos[o + j * kChunk + tid];
        b = row[y >> a.shift];
        off = y & (a.bs - 1);
        if (is_block(a, b)) e = exp_byte(exps[b]);
        else b = -1;
    }
    if (tid < kChunk) ex[tid] = (int16_t)e;
    // where each block goes
    if (tid >= MT - kChunk / 16 && ((tid - (MT - kChunk / 16)) << a.shift) < hi) {
        const int y = tid - (MT - kChunk / 16);
        const int64_t n = ((j << kChunkShift) >> a.shift) + y;
        int32_t t = -1;
        if (n >= x.y) {
            const int32_t r = a.rank[(o >> a.shift) + p + n];
            t = r >= 0 ? a.free_list[a.head[0].top - 1 - (x.w + r)] : row[n];
            if (!VALUES && r >= 0) a.taken[x.w + r] = t;
        }
        to[y] = is_block(a, t) ? t : -1;
    }
    if constexpr (!VALUES) {
        if (tid < kChunk) blk[tid] = b, info[tid] = off, top[tid] = 0;
        __syncthreads();
        const int per = a.dp / 16, n = hi * per;
        for (int i0 = lo * per + tid; i0 < n; i0 += 4 * MT) {
            uint4 z[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * MT, t = i < n ? i / per : lo;
                z[u] = make_uint4(0u, 0u, 0u, 0u);
                if (i < n && blk[t] >= 0) z[u] = *(const uint4 *)(codes + blk[t] * size + info[t] * a.dp + 16 * (i - t * per));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * MT;
                if (i >= n) break;
                *(uint4 *)(lds + 16 * i) = z[u];
                const uint32_t m = max_bytes(max_bytes(magnitudes(z[u].x), magnitudes(z[u].y)),
                                             max_bytes(magnitudes(z[u].z), magnitudes(z[u].w)));
                atomicMax(&top[i / per], max(max(m & 0xFFu, (m >> 8) & 0xFFu), max((m >> 16) & 0xFFu, m >> 24)));
            }
        }
    } else {
        for (int i = tid; i < a.dp * vrow / 16; i += MT) ((uint4 *)lds)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (tid < kChunk) place[tid] = make_int2(mine ? b : -2, off >> 6), stay[tid] = 0;
        __syncthreads();
        // the first token of a group stands for it
        const bool first = mine && (tid == lo || place[tid - 1].x != b || place[tid - 1].y != off >> 6);
        const uint64_t heads = __ballot(first);
        if (lane == 0 && w < kChunk / 64) s_count[w] = __popcll(heads);
        __syncthreads();
        int n = __popcll(heads & ((2ull << lane) - 1)) - 1, spans = 0;
#pragma unroll
        for (int i = 0; i < kChunk / 64; ++i) {
            if (i < w) n += s_count[i];
            spans += s_count[i];
        }
        if (first) blk[n] = b, info[n] = tid | off >> 6 << 8;
        if (mine) atomicOr((uint32_t *)&stay[n] + (off >> 5 & 1), 1u << (off & 31));
        __syncthreads();
        // a wave takes 64 rows of a group: `ppr` loads of 64 / ppr rows
        const int ppr = a.bs < 64 ? a.bs / 16 : 4, ps = __builtin_ctz(ppr), strips = (a.dp + 63) / 64;
        const int piece = lane & (ppr - 1);
        const uint32_t mine_at = (lane >> ps) * a.bs + 16 * piece;
        for (int y = w; y < spans * strips; y += MT / 64) {
            const int g = y / strips, r0 = 64 * (y - g * strips), bg = __builtin_amdgcn_readfirstlane(blk[g]);
            if (bg < 0) continue;
            const int in = __builtin_amdgcn_readfirstlane(info[g]);
            const uint64_t st = (uint64_t)__builtin_amdgcn_readfirstlane((int)(stay[g] >> 32)) << 32 |
                                (uint32_t)__builtin_amdgcn_readfirstlane((int)stay[g]);
            const uint8_t *from = a.vc + bg * size + 64 * (in >> 8) + (int64_t)r0 * a.bs;
            const uint32_t m = (uint32_t)(st >> (16 * piece)) & 0xFFFFu;
            const int rows = m ? a.dp - r0 - (lane >> ps) : 0;  // of this lane's, from the strip's first on
            uint4 z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[i] = make_uint4(0u, 0u, 0u, 0u);
                if (i < ppr && (i << (6 - ps)) < rows) z[i] = *(const uint4 *)(from + (i << (6 - ps)) * a.bs + mine_at);
            }
            const int at = (in & 0xFF) + __popcll(st & ((1ull << (16 * piece)) - 1));
            uint2 sel[4];
            bool full[4];
            int fill = at & 3;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint32_t nib = m >> (4 * v) & 15u;
                sel[v] = pack[nib << 2 | fill];
                fill += __popc(nib);
                full[v] = fill >= 4;
                fill &= 3;
            }
            const int out0 = (r0 + (lane >> ps)) * vrow + (at & ~3);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= ppr || (i << (6 - ps)) >= rows) continue;
                uint32_t *out = (uint32_t *)(lds + out0 + (i << (6 - ps)) * vrow), acc = 0;
                const uint32_t word[4] = {z[i].x, z[i].y, z[i].z, z[i].w};
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    acc = __builtin_amdgcn_perm(acc, word[v], sel[v].x);
                    if (full[v]) {
                        atomicOr(out, acc);
                        ++out;
                        acc = __builtin_amdgcn_perm(0u, word[v], sel[v].y);
                    }
                }
                if (fill) atomicOr(out, acc);
            }
        }
        __syncthreads();
        // the largest magnitude of every token: four tokens and a share of the rows a thread
        if (tid < kChunk) top[tid] = 0;
        __syncthreads();
        const int col = tid & (kChunk / 4 - 1);
        if (4 * col >= lo && 4 * col < hi) {
            uint32_t m = 0;
            for (int y = tid / (kChunk / 4); y < a.dp; y += MT / (kChunk / 4))
                m = max_bytes(m, magnitudes(*(const uint32_t *)(lds + y * vrow + 4 * col)));
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicMax(&top[4 * col + i], (m >> (8 * i)) & 0xFFu);
        }
    }
    __syncthreads();  // everything has been read
    if (tid == 0) __hip_atomic_store(&read[chunk], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (mine) atomicMax(&least[tid >> a.shift], least_exp((int)top[tid], e));
    __syncthreads();
    if (mine) ratio[tid] = exp_ratio(e, min(least[tid >> a.shift], 253));
    if (w == MT / 64 - 1) take_ticket();  // everyone has the one at hand
    // the chunks before this one that keep tokens of its positions
    {
        const int64_t r0 = a.within[chunk], r1 = (j + 1) * kChunk < x.x ? a.within[chunk + 1] : x.x;
        const int64_t i0 = max(r0, (int64_t)x.y * a.bs) >> kChunkShift, i1 = min((r1 + kChunk - 1) >> kChunkShift, j);
        int polls = 0;
        for (int64_t i = i0 + tid; i < i1; i += MT)
            while (!__hip_atomic_load(&read[t0 + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) && ++polls < a.polls)
                __builtin_amdgcn_s_sleep(1);
        if (polls >= a.polls && i0 + tid < i1) {  // in vain: what lies there may not have been read, so nothing is written
            for (int y = 0; y < kChunk / 16; ++y) to[y] = -1;
            a.refused[0] = -1;
        }
    }
    __syncthreads();
    uint8_t *dst = VALUES ? a.vc : a.kc;
    if constexpr (!VALUES) {
        const int per = a.dp / 16;
        for (int i = lo * per + tid; i < hi * per; i += MT) {
            const int t = i / per, n = to[t >> a.shift];
            if (n < 0) continue;
            const float f = ratio[t];
            uint4 z = *(const uint4 *)(lds + 16 * i);
            z.x = scale_codes(z.x, f, f, f, f), z.y = scale_codes(z.y, f, f, f, f);
            z.z = scale_codes(z.z, f, f, f, f), z.w = scale_codes(z.w, f, f, f, f);
            *(uint4 *)(dst + n * size + 16 * (i - (t >> a.shift << a.shift) * per)) = z;
        }
    } else {
        // a block's rows one after the other, 16 tokens a thread
        const int per = a.bs / 16, each = a.dp * per;
        for (int i = tid; i < each * (kChunk >> a.shift); i += MT) {
            const int n = i / each, in = i - n * each, y = in / per, t = (n << a.shift) + 16 * (in - y * per);
            if (t < lo || t >= hi || to[n] < 0) continue;
            uint32_t z[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float4 f = *(const float4 *)(ratio + t + 4 * u);
                z[u] = scale_codes(*(const uint32_t *)(lds + y * vrow + t + 4 * u), f.x, f.y, f.z, f.w);
            }
            uint8_t *q = dst + to[n] * size + 16 * in;
            if (t + 16 <= hi) {
                *(uint4 *)q = make_uint4(z[0], z[1], z[2], z[3]);
            } else {
                for (int u = 0; t + u < hi; ++u) q[u] = (uint8_t)(z[u / 4] >> (8 * (u % 4)));
            }
        }
    }
    if (tid < kChunk >> a.shift && (tid << a.shift) >= lo && (tid << a.shift) < hi && to[tid] >= 0)
        (VALUES ? a.v_exp : a.k_exp)[to[tid]] = (uint8_t)min(least[tid], 253);
    }
}

// Every other workgroup begins with values, the rest with keys (at the size above 5 us less than two of three).
// Whoever is out of tickets counts down the owners of the blocks that the listed cells leave.
// ONCE: there is a workgroup for every chunk's keys and one for its values, so none asks for a second ticket (16 cells of
// 4000 tokens that grow and are compacted: 38 us, with second tickets 42).
template <bool ONCE>
__global__ void __launch_bounds__(MT, 6) compact_move(PageArgs a) {
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ MoveShared sh;
    for (int i = 0; i < (ONCE ? 1 : 2); ++i) {
        if ((blockIdx.x % 2 != 0) != (i == 1)) move_chunks<true, ONCE>(a, lds, sh);
        else move_chunks<false, ONCE>(a, lds, sh);
    }
    for (int64_t p = blockIdx.x; p < a.P; p += gridDim.x) {
        const int4 x = a.plan[p];
        if (x.x < 0) continue;
        const int64_t c = cell_of(a, p), b0 = block0(a, p), now = nb(a, x.x), had = nb(a, length_of(a, c));
        const int32_t *row = a.table + c * a.W;
        for (int64_t j = (x.z > 0 ? x.y : now) + threadIdx.x; j < had; j += MT)
            if (j >= now || a.rank[b0 + j] >= 0) leave_block(a, row[j]);
    }
}

// The blocks that were left onto the stack; the workgroups behind write the listed cells' new tables and lengths.
__global__ void __launch_bounds__(WT) compact_finish(PageArgs a) {
    if (blockIdx.x < a.nruns) {
        collect_run(a, blockIdx.x);
        return;
    }
    const int64_t p = blockIdx.x - a.nruns;
    const int4 x = a.plan[p];
    if (x.x < 0) return;
    const int64_t c = cell_of(a, p), b0 = block0(a, p), now = nb(a, x.x), had = nb(a, length_of(a, c));
    int32_t *row = a.table + c * a.W;
    if (x.z > 0)
        for (int64_t j = x.y + threadIdx.x; j < now; j += WT) {
            const int32_t r = a.rank[b0 + j];
            if (r >= 0) row[j] = a.taken[x.w + r];
        }
    for (int64_t j = now + threadIdx.x; j < had; j += WT) row[j] = -1;
    __syncthreads();  // everyone has read the length
    if (threadIdx.x == 0) a.lens[c] = x.x;
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
// kind 0: release, 1: fork, 2: compact
size_t layout(PageArgs &a, int kind, void *ws) {
    PageLayout l{(char *)ws};
    a.nruns = (a.n_blocks + kRun - 1) / kRun;
    a.head = l.take<PageHead>(1);
    if (kind != 1) a.marks = l.take<uint16_t>(a.nruns * WT), a.counts = l.take<int32_t>(a.nruns);
    if (kind != 0) a.claim = l.take<int32_t>(a.C);
    a.plan = l.take<int4>(kind == 0 ? a.C : a.P);
    if (kind == 2) {
        a.chunks = a.n_kept / kChunk + a.P;
        a.rank = l.take<int32_t>(a.n_kept / a.bs + a.P), a.taken = l.take<int32_t>(a.n_kept / a.bs + a.P);
        a.owner = l.take<int32_t>(a.chunks);
        a.within = l.take<int32_t>(a.chunks), a.read = l.take<int32_t>(2 * a.chunks);
        a.tickets = l.take<int32_t>(2 * kQueues * kApart);
        a.starts = l.take<int32_t>(kQueues + 1);
    }
    return align_up(l.off, 256);
}

PageArgs page_args(const fw_cache &cache, const fw_cells &cells) {
    PageArgs a{};
    a.C = cells.C, a.W = cells.max_blocks, a.n_blocks = cache.n_blocks;
    a.bs = cache.block_size, a.shift = __builtin_ctz(cache.block_size), a.dp = cache_row(cache.d);
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
    if (a.nruns > kFewRuns) hipLaunchKernelGGL(clear_all, dim3((unsigned)std::min<int64_t>(a.nruns / 4 + 1, 1024)), dim3(WT), 0, st, a);
    hipLaunchKernelGGL(release_plan, dim3(1), dim3(PT), 0, st, a);
    hipLaunchKernelGGL(release_apply, dim3((unsigned)a.C), dim3(WT), 0, st, a);
    if (a.nruns > kFewRuns) hipLaunchKernelGGL(count_runs, dim3((unsigned)a.nruns), dim3(WT), 0, st, a);
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

// kPolls, but for the test that sets 0: then every wait is given up.  No part of the interface.
extern "C" {
int32_t fw_compact_polls = kPolls;
}

hipError_t launch_cell_compact(const fw_cache &cache, const fw_cells &cells, int64_t P, const int32_t *which,
                               const int64_t *offsets, int64_t n_kept, const int32_t *kept_pos, int32_t *refused,
                               void *ws, hipStream_t st) {
    PageArgs a = page_args(cache, cells);
    a.P = P, a.which = which, a.offsets = offsets, a.n_kept = n_kept, a.kept_pos = kept_pos, a.refused = refused;
    a.polls = fw_compact_polls;
    layout(a, 2, ws);
    if (P > 0) hipLaunchKernelGGL(compact_check, dim3((unsigned)P), dim3(CT), 0, st, a);
    hipLaunchKernelGGL(compact_plan, dim3(1), dim3(PT), 0, st, a);
    if (P == 0) return hipGetLastError();
    const unsigned lds = a.dp * (kChunk + 4);
    if (2 * a.chunks <= kMovers) hipLaunchKernelGGL(compact_move<true>, dim3((unsigned)(2 * a.chunks)), dim3(MT), lds, st, a);
    else hipLaunchKernelGGL(compact_move<false>, dim3(kMovers), dim3(MT), lds, st, a);
    if (a.nruns > kFewRuns) hipLaunchKernelGGL(count_runs, dim3((unsigned)a.nruns), dim3(WT), 0, st, a);
    hipLaunchKernelGGL(compact_finish, dim3((unsigned)(a.nruns + P)), dim3(WT), 0, st, a);
    return hipGetLastError();
}

}  // namespace fw
