// C ABI of libfw: argument validation, workspace layout and launch order.
// No entry point allocates device memory, synchronises or copies to the host.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <mutex>

#include "fw_internal.hpp"

// Scratch space of fw_dense_topk_noalloc: one copy per GPU, allocated with the
// code object and held until the process ends.  In host code this name only
// stands in for the symbol; kernels and copies use the per-device address
// taken from hipGetSymbolAddress below, never the name itself.
static __device__ __align__(256) unsigned char scratch[FW_NOALLOC_SCRATCH_BYTES];

namespace {

thread_local char g_err[512] = "";

fw_status fail(fw_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return s;
}

fw_status hip_status(hipError_t e, const char *where) {
    if (e == hipSuccess) return FW_OK;
    return fail(FW_E_HIP, "%s: %s", where, hipGetErrorString(e));
}

// Sequential carve-out of the caller's workspace in 256-byte aligned pieces.
struct Carve {
    char *base;
    size_t off = 0;
    explicit Carve(void *b) : base((char *)b) {}
    template <typename T> T *take(size_t count) {
        off = fw::align_up(off, 256);
        T *p = base ? (T *)(base + off) : nullptr;
        off += count * sizeof(T);
        return p;
    }
    size_t size() const { return fw::align_up(off, 256); }
};

fw_status check_rows(const fw_rows *rows, bool need_v) {
    if (!rows) return fail(FW_E_NULL, "rows is NULL");
    if (rows->dtype != FW_F32 && rows->dtype != FW_BF16)
        return fail(FW_E_DTYPE, "unknown dtype %d", (int)rows->dtype);
    if (!rows->q || !rows->k) return fail(FW_E_NULL, "rows->q or rows->k is NULL");
    if (need_v && !rows->v) return fail(FW_E_NULL, "rows->v is NULL");
    if (rows->H < 1 || rows->G < 1 || rows->n < 1)
        return fail(FW_E_SHAPE, "H, G, n must be >= 1 (H=%lld G=%lld n=%lld)", (long long)rows->H,
                    (long long)rows->G, (long long)rows->n);
    if (rows->d < 1 || rows->d > 256) return fail(FW_E_SHAPE, "d must be in [1, 256], got %lld", (long long)rows->d);
    if (rows->n > (1ll << 30)) return fail(FW_E_SHAPE, "n must be <= 2^30");
    if (rows->H > (1ll << 31) / rows->G) return fail(FW_E_SHAPE, "H*G must be < 2^31");
    const double hgn = (double)rows->H * (double)rows->G * (double)rows->n;
    if (hgn >= 1099511627776.0) return fail(FW_E_SHAPE, "H*G*n must be < 2^40");
    return FW_OK;
}

fw_status check_ws(void *ws, size_t ws_bytes, size_t need) {
    if (need && !ws) return fail(FW_E_WORKSPACE, "workspace is NULL, %zu bytes needed", need);
    if (ws_bytes < need) return fail(FW_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    return FW_OK;
}

// ---------------------------------------------------------------------------
// fw_dense_topk
// ---------------------------------------------------------------------------
fw_status parse_ks(const fw_rows *rows, const int32_t *ks, int32_t n_ks, fw::KsArg *out) {
    if (!ks) return fail(FW_E_NULL, "ks is NULL");
    if (n_ks < 1 || n_ks > FW_MAX_KS) return fail(FW_E_SHAPE, "n_ks must be in [1, %d]", FW_MAX_KS);
    int idx[FW_MAX_KS];
    for (int i = 0; i < n_ks; ++i) {
        if (ks[i] < 1 || ks[i] > rows->n)
            return fail(FW_E_SHAPE, "ks[%d] = %d outside [1, n=%lld]", i, ks[i], (long long)rows->n);
        idx[i] = i;
    }
    std::sort(idx, idx + n_ks, [&](int a, int b) { return ks[a] < ks[b]; });
    out->n = n_ks;
    for (int t = 0; t < n_ks; ++t) {
        if (t && ks[idx[t]] == ks[idx[t - 1]]) return fail(FW_E_SHAPE, "ks must be distinct");
        out->k[t] = ks[idx[t]];
        out->perm[t] = idx[t];
    }
    for (int t = n_ks; t < FW_MAX_KS; ++t) { out->k[t] = 0; out->perm[t] = 0; }
    return FW_OK;
}

struct DenseTopkWs {
    float *z, *row_m, *row_l;
    uint32_t *thr_key;
    int32_t *thr_cut;
    int splits;           // key ranges of the tier sums
    float *part, *part_m; // their partial sums, splits > 1
    size_t bytes;
};

DenseTopkWs dense_topk_layout(const fw_rows *rows, int n_ks, void *ws) {
    Carve c(ws);
    const size_t R = (size_t)rows->H * rows->G;
    DenseTopkWs w;
    w.z = c.take<float>(R * rows->n);
    w.row_m = c.take<float>(R);
    w.row_l = c.take<float>(R);
    w.thr_key = c.take<uint32_t>(R * n_ks);
    w.thr_cut = c.take<int32_t>(R * n_ks);
    // Partial sums only as far as a call that fits the static scratch array
    // without them still fits it with them.
    const size_t base = c.size(), nt = (size_t)n_ks + 1;
    const auto extra = [&](int s) {
        return fw::align_up((size_t)s * R * nt * rows->d * sizeof(float), 256) +
               fw::align_up((size_t)s * R * nt * sizeof(float), 256);
    };
    w.splits = fw::tiers_splits(rows->dtype, rows->H, rows->G, rows->n);
    while (w.splits > 1 && base <= FW_NOALLOC_SCRATCH_BYTES && base + extra(w.splits) > FW_NOALLOC_SCRATCH_BYTES)
        --w.splits;
    w.part = w.part_m = nullptr;
    if (w.splits > 1) {
        w.part = c.take<float>((size_t)w.splits * R * nt * rows->d);
        w.part_m = c.take<float>((size_t)w.splits * R * nt);
    }
    w.bytes = c.size();
    return w;
}

// ---------------------------------------------------------------------------
// argument checks of the other entry points
// ---------------------------------------------------------------------------
fw_status check_best_subset(const fw_rows *rows, int32_t k) {
    fw_status s = check_rows(rows, true);
    if (s != FW_OK) return s;
    if (k < 1 || k > rows->n) return fail(FW_E_SHAPE, "k = %d outside [1, n=%lld]", k, (long long)rows->n);
    if (rows->n > 64) return fail(FW_E_UNSUPPORTED, "exhaustive enumeration needs n <= 64 (n=%lld)", (long long)rows->n);
    if (fw::binom((int)rows->n, k) >= (1ull << 31))
        return fail(FW_E_UNSUPPORTED, "C(n=%lld, k=%d) must be < 2^31", (long long)rows->n, k);
    if (!fw::best_subset_plannable(rows->n, k))
        return fail(FW_E_UNSUPPORTED, "no enumeration plan fits for n=%lld, k=%d", (long long)rows->n, k);
    return FW_OK;
}

fw_status check_swap(const fw_rows *rows, int32_t k, int32_t max_iters) {
    fw_status s = check_rows(rows, true);
    if (s != FW_OK) return s;
    if (k < 1 || k > rows->n) return fail(FW_E_SHAPE, "k = %d outside [1, n=%lld]", k, (long long)rows->n);
    if (max_iters < 0 || max_iters > 4096) return fail(FW_E_SHAPE, "max_iters must be in [0, 4096]");
    if (rows->n > 64 && rows->H * rows->G > 65535)
        return fail(FW_E_UNSUPPORTED, "rows longer than 64 keys: at most 65535 rows per call");
    return FW_OK;
}

fw_status check_compact(int32_t dtype, const void *k, const void *v, int64_t H, int64_t hpl, int64_t n,
                        int64_t d, const float *importance, int64_t budget, int32_t floor, int64_t cap) {
    if (dtype != FW_F32 && dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)dtype);
    if (!k || !v || !importance) return fail(FW_E_NULL, "k, v and importance are required");
    if (H < 1 || n < 1 || d < 1 || d > 4096) return fail(FW_E_SHAPE, "need H >= 1, n >= 1, 1 <= d <= 4096");
    if (n > (1ll << 30) || (double)H * (double)n >= 1099511627776.0) return fail(FW_E_SHAPE, "H*n too large");
    if (hpl < 1 || H % hpl != 0) return fail(FW_E_SHAPE, "heads_per_layer must divide H");
    if (floor < 0) return fail(FW_E_SHAPE, "recency_floor must be >= 0");
    const int64_t f = floor < n ? floor : n;
    if (cap < 0 || (cap > 0 && cap < f))
        return fail(FW_E_SHAPE, "cap must be 0 (none) or >= min(recency_floor, n), got %lld", (long long)cap);
    const int64_t per_cell = (cap > 0 && cap < n) ? cap : n;
    if (budget < H * f || budget > H * per_cell)
        return fail(FW_E_SHAPE, "budget_entries %lld outside [H*floor, H*min(cap, n)] = [%lld, %lld]",
                    (long long)budget, (long long)(H * f), (long long)(H * per_cell));
    if (budget >= (1ll << 31)) return fail(FW_E_SHAPE, "budget_entries must be < 2^31");
    return FW_OK;
}

fw_status check_pool(const fw_rows *rows, int32_t n_budgets, const int32_t *s, const int32_t *extra,
                     int32_t max_swaps) {
    fw_status st = check_rows(rows, true);
    if (st != FW_OK) return st;
    if (!s || !extra) return fail(FW_E_NULL, "s and extra are required");
    if (n_budgets < 1 || n_budgets > FW_POOL_MAX_BUDGETS)
        return fail(FW_E_SHAPE, "n_budgets must be in [1, %d]", FW_POOL_MAX_BUDGETS);
    for (int b = 0; b < n_budgets; ++b) {
        if (s[b] < 1 || extra[b] < 0 || (int64_t)s[b] + extra[b] > rows->n)
            return fail(FW_E_SHAPE, "budget %d: need 1 <= s, 0 <= extra, s + extra <= n (s=%d extra=%d n=%lld)", b,
                        s[b], extra[b], (long long)rows->n);
        if (s[b] + extra[b] > 64) return fail(FW_E_UNSUPPORTED, "budget %d: s + extra = %d > 64 pool keys", b, s[b] + extra[b]);
    }
    if (max_swaps < 0 || max_swaps > 4096) return fail(FW_E_SHAPE, "max_swaps must be in [0, 4096]");
    if (rows->n > 8192) return fail(FW_E_UNSUPPORTED, "n = %lld > 8192 for the candidate-set search", (long long)rows->n);
    if (!fw::pool_plannable(rows->n, (int)rows->d, n_budgets, s, extra))
        return fail(FW_E_UNSUPPORTED, "no enumeration plan for these budgets within the limits");
    return FW_OK;
}

}  // namespace

extern "C" {

const char *fw_last_error(void) { return g_err; }
const char *fw_version(void) { return "libfw 0.1 (gfx950)"; }

size_t dense_topk_ws_bytes(const fw_rows *rows, const fw::KsArg &k) {
    if (fw::mp_topk_supported(*rows, k) || fw::fused_topk_supported(*rows, k))
        return fw::fused_topk_ws_bytes(*rows, k.k[k.n - 1]);
    return dense_topk_layout(rows, k.n, nullptr).bytes;
}

size_t fw_dense_topk_workspace_size(const fw_rows *rows, const int32_t *ks, int32_t n_ks) {
    fw::KsArg k;
    if (check_rows(rows, true) != FW_OK || parse_ks(rows, ks, n_ks, &k) != FW_OK) return 0;
    return dense_topk_ws_bytes(rows, k);
}

}  // extern "C"

namespace {

fw_status check_dense_topk(const fw_rows *rows, const int32_t *ks, int32_t n_ks, const float *gap,
                           const float *dropped, const int32_t *topk_idx, fw::KsArg *k) {
    fw_status s = check_rows(rows, true);
    if (s != FW_OK) return s;
    if ((s = parse_ks(rows, ks, n_ks, k)) != FW_OK) return s;
    if (!gap || !dropped) return fail(FW_E_NULL, "gap and dropped are required");
    if (topk_idx && k->k[k->n - 1] > 16384) return fail(FW_E_UNSUPPORTED, "topk_idx needs kmax <= 16384");
    return FW_OK;
}

// Launches of fw_dense_topk once the arguments and the workspace are checked.
fw_status dense_topk_launch(const fw_rows *rows, const fw::KsArg &k, float *o, float *o_s, float *gap,
                            float *dropped, int32_t *topk_idx, void *ws, hipStream_t st) {
    const int kmax = k.k[k.n - 1];
    const int n_ks = k.n;
    if (fw::mp_topk_supported(*rows, k))
        return hip_status(fw::launch_mp_topk(*rows, k, o, o_s, gap, dropped, topk_idx, ws, st), "fw_dense_topk");
    if (fw::fused_topk_supported(*rows, k))
        return hip_status(fw::launch_fused_topk(*rows, k, o, o_s, gap, dropped, topk_idx, ws, st),
                          "fw_dense_topk");
    const DenseTopkWs w = dense_topk_layout(rows, n_ks, ws);
    const int64_t H = rows->H, G = rows->G, n = rows->n;
    const int d = (int)rows->d;
    hipError_t e = fw::launch_scores(rows->dtype, rows->q, rows->k, rows->scale, rows->bias, H, G, n,
                                     d, w.z, st);
    if (e == hipSuccess)
        e = fw::launch_select(w.z, H * G, n, k, w.row_m, w.row_l, w.thr_key, w.thr_cut, topk_idx,
                              kmax, st);
    if (e == hipSuccess)
        e = fw::launch_tiers(rows->dtype, rows->v, w.z, w.row_m, w.row_l, w.thr_key, w.thr_cut, H, G, n, d, k, o,
                             o_s, gap, dropped, w.splits, w.part, w.part_m, st);
    return hip_status(e, "fw_dense_topk");
}

// Per-device address of `scratch`, taken once per device with that device
// current (every GPU holds its own copy at its own address).
constexpr int kScratchDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch_ptr[kScratchDevices];

fw_status scratch_address(hipStream_t st, void **out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_status(e, "fw_dense_topk_noalloc: hipGetDevice");
    if (st) {
        int sdev = -1;
        if ((e = hipStreamGetDevice(st, &sdev)) != hipSuccess)
            return hip_status(e, "fw_dense_topk_noalloc: hipStreamGetDevice");
        if (sdev != dev)
            return fail(FW_E_UNSUPPORTED, "stream belongs to device %d but device %d is current", sdev, dev);
    }
    if (dev < 0 || dev >= kScratchDevices)
        return fail(FW_E_UNSUPPORTED, "device %d is beyond the %d devices the scratch table holds", dev,
                    kScratchDevices);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void *p = nullptr;
        if ((e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch))) != hipSuccess)
            return hip_status(e, "fw_dense_topk_noalloc: hipGetSymbolAddress");
        if (!p) return fail(FW_E_HIP, "fw_dense_topk_noalloc: no device address for the scratch array");
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return FW_OK;
}

}  // namespace

extern "C" {

fw_status fw_dense_topk(const fw_rows *rows, const int32_t *ks, int32_t n_ks, float *o, float *o_s,
                        float *gap, float *dropped, int32_t *topk_idx, void *ws, size_t ws_bytes,
                        fw_stream stream) {
    fw::KsArg k;
    fw_status s = check_dense_topk(rows, ks, n_ks, gap, dropped, topk_idx, &k);
    if (s != FW_OK) return s;
    if ((s = check_ws(ws, ws_bytes, dense_topk_ws_bytes(rows, k))) != FW_OK) return s;
    return dense_topk_launch(rows, k, o, o_s, gap, dropped, topk_idx, ws, (hipStream_t)stream);
}

fw_status fw_dense_topk_noalloc(const fw_rows *rows, const int32_t *ks, int32_t n_ks, float *o, float *o_s,
                                float *gap, float *dropped, int32_t *topk_idx, fw_stream stream) {
    fw::KsArg k;
    fw_status s = check_dense_topk(rows, ks, n_ks, gap, dropped, topk_idx, &k);
    if (s != FW_OK) return s;
    const size_t need = dense_topk_ws_bytes(rows, k);
    if (need > FW_NOALLOC_SCRATCH_BYTES)
        return fail(FW_E_UNSUPPORTED,
                    "fw_dense_topk_noalloc: this call needs %zu bytes of scratch, more than the %zu the "
                    "library holds per device (use fw_dense_topk with a workspace)",
                    need, (size_t)FW_NOALLOC_SCRATCH_BYTES);
    hipStream_t st = (hipStream_t)stream;
    void *ws = nullptr;
    if ((s = scratch_address(st, &ws)) != FW_OK) return s;
    return dense_topk_launch(rows, k, o, o_s, gap, dropped, topk_idx, ws, st);
}

// ---------------------------------------------------------------------------
size_t fw_best_subset_workspace_size(const fw_rows *rows, int32_t k) {
    if (check_best_subset(rows, k) != FW_OK) return 0;
    return fw::best_subset_ws_bytes(rows->n, k);
}

fw_status fw_best_subset(const fw_rows *rows, int32_t k, int32_t *best_idx, float *best_gap,
                         float *topk_gap, float *closed, float *dropped_topk, int32_t *topk_idx,
                         void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status s = check_best_subset(rows, k);
    if (s != FW_OK) return s;
    if (!best_idx || !best_gap) return fail(FW_E_NULL, "best_idx and best_gap are required");
    if ((s = check_ws(ws, ws_bytes, fw::best_subset_ws_bytes(rows->n, k))) != FW_OK) return s;
    hipError_t e = fw::launch_best_subset(*rows, k, best_idx, best_gap, topk_gap, closed,
                                          dropped_topk, topk_idx, ws, (hipStream_t)stream);
    return hip_status(e, "fw_best_subset");
}

// ---------------------------------------------------------------------------
size_t fw_pool_subset_workspace_size(const fw_rows *rows, int32_t n_budgets, const int32_t *s,
                                     const int32_t *extra) {
    if (check_pool(rows, n_budgets, s, extra, 0) != FW_OK) return 0;
    return fw::pool_ws_bytes(*rows, n_budgets, s, extra);
}

fw_status fw_pool_subset(const fw_rows *rows, int32_t n_budgets, const int32_t *s, const int32_t *extra,
                         int32_t max_swaps, int32_t fw_iters, int32_t *pool_idx, int32_t *best_idx,
                         int32_t *bal_idx, int32_t *geo_idx, int32_t *n_swaps, float *stats, float flat_threshold,
                         float *cell_median, uint8_t *cell_flat, void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status st = check_pool(rows, n_budgets, s, extra, max_swaps);
    if (st != FW_OK) return st;
    if (fw_iters < 0 || fw_iters > 4096) return fail(FW_E_SHAPE, "fw_iters must be in [0, 4096]");
    if (!best_idx || !stats) return fail(FW_E_NULL, "best_idx and stats are required");
    if ((st = check_ws(ws, ws_bytes, fw::pool_ws_bytes(*rows, n_budgets, s, extra))) != FW_OK) return st;
    hipError_t e = fw::launch_pool(*rows, n_budgets, s, extra, max_swaps, fw_iters, pool_idx, best_idx, bal_idx,
                                   geo_idx, n_swaps, stats, flat_threshold, cell_median, cell_flat, ws,
                                   (hipStream_t)stream);
    return hip_status(e, "fw_pool_subset");
}

// ---------------------------------------------------------------------------
size_t fw_swap_workspace_size(const fw_rows *rows, int32_t k, int32_t max_iters) {
    if (check_swap(rows, k, max_iters) != FW_OK) return 0;
    return fw::swap_ws_bytes(*rows, k, max_iters);
}

fw_status fw_swap(const fw_rows *rows, int32_t k, int32_t max_iters, int32_t *s_idx, float *gap_traj,
                  int32_t *n_swaps, float *dropped, void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status s = check_swap(rows, k, max_iters);
    if (s != FW_OK) return s;
    if (!s_idx || !gap_traj || !n_swaps) return fail(FW_E_NULL, "s_idx, gap_traj and n_swaps are required");
    if ((s = check_ws(ws, ws_bytes, fw::swap_ws_bytes(*rows, k, max_iters))) != FW_OK) return s;
    hipError_t e = fw::launch_swap(*rows, k, max_iters, s_idx, gap_traj, n_swaps, dropped, ws,
                                   (hipStream_t)stream);
    return hip_status(e, "fw_swap");
}

// ---------------------------------------------------------------------------
size_t fw_dropped_mass_curve_workspace_size(const fw_rows *rows) {
    if (check_rows(rows, false) != FW_OK) return 0;
    return fw::curve_ws_bytes(*rows);
}

fw_status fw_dropped_mass_curve(const fw_rows *rows, float *importance, float *curve, int32_t *order,
                                void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status s = check_rows(rows, false);
    if (s != FW_OK) return s;
    if (!importance || !curve) return fail(FW_E_NULL, "importance and curve are required");
    if ((s = check_ws(ws, ws_bytes, fw::curve_ws_bytes(*rows))) != FW_OK) return s;
    hipError_t e = fw::launch_curve(*rows, importance, curve, order, ws, (hipStream_t)stream);
    return hip_status(e, "fw_dropped_mass_curve");
}

// ---------------------------------------------------------------------------
size_t fw_ragged_compact_workspace_size(int64_t H, int64_t n, int64_t d, int64_t budget_entries) {
    if (H < 1 || n < 1 || d < 1 || budget_entries < 0) return 0;
    return fw::compact_ws_bytes(H, n);
}

fw_status fw_ragged_compact(int32_t dtype, const void *k, const void *v, int64_t H, int64_t heads_per_layer,
                            int64_t n, int64_t d, const float *importance, int64_t budget_entries,
                            int32_t recency_floor, int64_t cap, int64_t *offsets, int32_t *kept_pos,
                            void *k_out, void *v_out, float *tau, float *dropped, int64_t *bytes_held, void *ws,
                            size_t ws_bytes, fw_stream stream) {
    fw_status s = check_compact(dtype, k, v, H, heads_per_layer, n, d, importance, budget_entries,
                                recency_floor, cap);
    if (s != FW_OK) return s;
    if (!offsets || !kept_pos || !k_out || !v_out)
        return fail(FW_E_NULL, "offsets, kept_pos, k_out and v_out are required");
    if ((s = check_ws(ws, ws_bytes, fw::compact_ws_bytes(H, n))) != FW_OK) return s;
    hipError_t e = fw::launch_compact(dtype, k, v, H, heads_per_layer, n, d, importance,
                                      budget_entries, recency_floor, cap, offsets, kept_pos, k_out, v_out,
                                      tau, dropped, bytes_held, ws, (hipStream_t)stream);
    return hip_status(e, "fw_ragged_compact");
}

fw_status fw_maxpool_scores(const float *scores, int64_t H, int64_t n, int32_t kernel, float *out,
                            fw_stream stream) {
    if (!scores || !out) return fail(FW_E_NULL, "scores and out are required");
    if (H < 1 || n < 1 || (double)H * (double)n >= 1099511627776.0) return fail(FW_E_SHAPE, "need H, n >= 1, H*n < 2^40");
    if (kernel < 1 || kernel % 2 == 0 || kernel > 1023) return fail(FW_E_SHAPE, "kernel must be odd, 1..1023");
    if (scores == out && kernel > 1) return fail(FW_E_SHAPE, "out must not alias scores");
    return hip_status(fw::launch_maxpool(scores, H, n, kernel, out, (hipStream_t)stream), "fw_maxpool_scores");
}

// ---------------------------------------------------------------------------
size_t fw_group_vote_workspace_size(const fw_rows *rows, int32_t s, int32_t group_size) {
    (void)rows;
    (void)s;
    (void)group_size;
    return 0;
}

fw_status fw_group_vote(const fw_rows *rows, int32_t s, int32_t group_size, int32_t *vote_idx, float *es_vote,
                        float *es_top, float *dropped, void *ws, size_t ws_bytes, fw_stream stream) {
    (void)ws;
    (void)ws_bytes;
    fw_status st = check_rows(rows, true);
    if (st != FW_OK) return st;
    if (group_size < 1 || rows->G % group_size != 0)
        return fail(FW_E_SHAPE, "group_size must divide G (G=%lld group_size=%d)", (long long)rows->G, group_size);
    if (s < 1 || s > rows->n) return fail(FW_E_SHAPE, "s must be in [1, n=%lld], got %d", (long long)rows->n, s);
    if (s > 256) return fail(FW_E_UNSUPPORTED, "s = %d > 256", s);
    if (!fw::vote_supported(*rows, s, group_size))
        return fail(FW_E_UNSUPPORTED, "n, d and the group size need more than 160 KiB of LDS");
    if (!vote_idx || !es_vote || !es_top) return fail(FW_E_NULL, "vote_idx, es_vote and es_top are required");
    hipError_t e = fw::launch_vote(*rows, s, group_size, vote_idx, es_vote, es_top, dropped, (hipStream_t)stream);
    return hip_status(e, "fw_group_vote");
}

}  // extern "C"


// ---------------------------------------------------------------------------
// serving: prompt attention, block tables, the 8-bit cache
// ---------------------------------------------------------------------------
namespace {

fw_status check_packed(const fw_packed *p) {
    if (!p) return fail(FW_E_NULL, "packed is NULL");
    if (p->dtype != FW_F32 && p->dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)p->dtype);
    if (p->B < 1 || p->Hkv < 1 || p->Hq < 1 || p->Tq < 0 || p->Tk < 0)
        return fail(FW_E_SHAPE, "need B, Hq, Hkv >= 1 and Tq, Tk >= 0 (B=%lld Hq=%lld Hkv=%lld Tq=%lld Tk=%lld)",
                    (long long)p->B, (long long)p->Hq, (long long)p->Hkv, (long long)p->Tq, (long long)p->Tk);
    if (p->Hq % p->Hkv != 0)
        return fail(FW_E_SHAPE, "Hkv must divide Hq (Hq=%lld Hkv=%lld)", (long long)p->Hq, (long long)p->Hkv);
    if (p->d < 1 || p->d > 256) return fail(FW_E_SHAPE, "d must be in [1, 256], got %lld", (long long)p->d);
    constexpr int64_t most = (int64_t)1 << 31;
    if (p->Hq >= most || p->Tq >= most || p->Tk > (1ll << 30) || p->B >= most || p->Tq * p->Hq >= most)
        return fail(FW_E_SHAPE, "need Tq*Hq < 2^31, Tk <= 2^30 and B < 2^31");
    // one workgroup of 256 threads per row tile and key/value head, 64 rows or more to a tile; a grid holds fewer than 2^32 threads
    if ((p->Tq * (p->Hq / p->Hkv) / 64 + 1 + p->B) >= ((int64_t)1 << 24) / p->Hkv)
        return fail(FW_E_SHAPE, "too many sequences and heads for one call");
    // every workgroup looks through the sequences for its own: 65,536 sequences of one position and 8 heads take 157
    // ms, a quarter of them 11, and 2^23 of one head would hold the GPU for minutes
    if ((p->Tq * (p->Hq / p->Hkv) / 64 + 1 + p->B) * p->Hkv >= ((int64_t)1 << 36) / p->B)
        return fail(FW_E_SHAPE, "(Tq*Hq/Hkv/64 + 1 + B)*Hkv * B must be < 2^36");
    const int64_t strides[] = {p->q_row, p->q_head, p->k_row, p->k_head, p->v_row, p->v_head};
    for (int64_t s : strides)
        if (s < 0 || s >= most) return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (!p->cu_q || !p->cu_k) return fail(FW_E_NULL, "cu_q and cu_k are required");
    if (p->Tq > 0 && !p->q) return fail(FW_E_NULL, "q is NULL");
    if (p->Tk > 0 && (!p->k || !p->v)) return fail(FW_E_NULL, "k or v is NULL");
    return FW_OK;
}

struct PromptWs {
    int splits;
    float *part_o, *part_lse;
    size_t bytes;
};
PromptWs prompt_layout(const fw_packed &p, void *ws) {
    PromptWs w{};
    w.splits = fw::prompt_splits(p);
    if (w.splits > 1) {
        Carve c(ws);
        const size_t rows = (size_t)w.splits * p.Tq * p.Hq;
        w.part_o = c.take<float>(rows * p.d);
        w.part_lse = c.take<float>(rows);
        w.bytes = c.size();
    }
    return w;
}

fw_status check_block(int32_t block_size) {
    if (block_size < 16 || block_size > 256 || (block_size & (block_size - 1)))
        return fail(FW_E_SHAPE, "block_size must be a power of two in [16, 256], got %d", (int)block_size);
    return FW_OK;
}

fw_status check_cache(const fw_cache *c) {
    if (!c) return fail(FW_E_NULL, "cache is NULL");
    if (!c->k || !c->v || !c->k_exp || !c->v_exp) return fail(FW_E_NULL, "cache->k, v, k_exp and v_exp are required");
    if ((uintptr_t)c->k % 16 || (uintptr_t)c->v % 16) return fail(FW_E_SHAPE, "cache->k and v must be 16-byte aligned");
    if (c->d < 1 || c->d > 256) return fail(FW_E_SHAPE, "d must be in [1, 256], got %lld", (long long)c->d);
    if (c->n_blocks < 1 || c->n_blocks >= ((int64_t)1 << 31)) return fail(FW_E_SHAPE, "n_blocks must be in [1, 2^31)");
    return check_block(c->block_size);
}

fw_status check_decode(int32_t block_size, int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t max_blocks) {
    if (S < 1 || T < 1 || Hq < 1 || Hkv < 1 || max_blocks < 1)
        return fail(FW_E_SHAPE, "S, T, Hq, Hkv and max_blocks must be >= 1");
    // a grid holds fewer than 2^32 threads: up to 512 for a cell, 64 for a row
    constexpr int64_t m31 = (int64_t)1 << 31, m26 = (int64_t)1 << 26, m22 = (int64_t)1 << 22;
    if (S >= m22 || Hkv >= m22 || S * Hkv >= m22) return fail(FW_E_SHAPE, "S*Hkv must be < 2^22");
    if (Hq % Hkv != 0) return fail(FW_E_SHAPE, "Hkv must divide Hq (Hq=%lld Hkv=%lld)", (long long)Hq, (long long)Hkv);
    if (T > 4096 || Hq / Hkv > 4096 || T * (Hq / Hkv) > 4096) return fail(FW_E_SHAPE, "T*Hq/Hkv must be <= 4096");
    // decode_join: four rows to a workgroup of 256 threads
    if (S * Hkv * (T * (Hq / Hkv)) > m26 - 4) return fail(FW_E_SHAPE, "S*T*Hq must be <= 2^26 - 4");
    if (max_blocks >= m31 / block_size) return fail(FW_E_SHAPE, "max_blocks * block_size must be < 2^31");
    if ((double)(S * Hkv) * (double)(max_blocks * block_size) >= 68719476736.0)
        return fail(FW_E_SHAPE, "S*Hkv * max_blocks * block_size must be < 2^36");
    return FW_OK;
}

// rows [T][H][d] that a call writes: none may meet another
bool rows_apart(int64_t T, int64_t H, int64_t d, int64_t row, int64_t head) {
    if (T == 0 || H == 0) return true;
    const bool heads_inside = (H == 1 || head >= d) && (T == 1 || row >= (H - 1) * head + d);
    const bool rows_inside = (T == 1 || row >= d) && (H == 1 || head >= (T - 1) * row + d);
    return heads_inside || rows_inside;
}

fw_status check_heads(const fw_heads *h) {
    if (!h) return fail(FW_E_NULL, "heads is NULL");
    if (h->dtype != FW_F32 && h->dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)h->dtype);
    constexpr int64_t m31 = (int64_t)1 << 31, m30 = (int64_t)1 << 30;
    if (h->T < 0 || h->Hq < 0 || h->Hkv < 0) return fail(FW_E_SHAPE, "T, Hq and Hkv must be >= 0");
    // a workgroup of 256 threads takes T / 2^23 tokens or more, at most eight; a grid holds fewer than 2^32 threads
    if (h->T > ((int64_t)1 << 25)) return fail(FW_E_SHAPE, "T must be <= 2^25, got %lld", (long long)h->T);
    if (h->Hq >= m30 || h->Hkv >= m30 || (h->T > 0 && h->Hq + h->Hkv >= m30 / h->T))
        return fail(FW_E_SHAPE, "T * (Hq + Hkv) must be < 2^30");
    if (h->d < 1 || h->d > 256) return fail(FW_E_SHAPE, "d must be in [1, 256], got %lld", (long long)h->d);
    if (h->rot < 0 || h->rot > h->d || h->rot % 2)
        return fail(FW_E_SHAPE, "rot must be even and in [0, d], got %lld", (long long)h->rot);
    const int64_t strides[] = {h->q_row, h->q_head, h->k_row, h->k_head};
    for (int64_t s : strides)
        if (s < 0 || s >= m31) return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (h->norm && !(h->eps >= 0.f)) return fail(FW_E_SHAPE, "eps must be >= 0");
    if (h->norm && (h->q_weight || h->k_weight) && h->w_dtype != FW_F32 && h->w_dtype != FW_BF16)
        return fail(FW_E_DTYPE, "unknown w_dtype %d", (int)h->w_dtype);
    if (h->T == 0) return FW_OK;
    if ((h->Hq > 0 && !h->q) || (h->Hkv > 0 && !h->k)) return fail(FW_E_NULL, "q or k is NULL");
    if (h->rot > 0 && (!h->pos || !h->freq)) return fail(FW_E_NULL, "pos and freq are required");
    return FW_OK;
}

fw_status check_cells(const fw_cache *cache, const fw_cells *t) {
    fw_status s = check_cache(cache);
    if (s != FW_OK) return s;
    if (!t) return fail(FW_E_NULL, "cells is NULL");
    if (t->C < 1 || t->C >= ((int64_t)1 << 22)) return fail(FW_E_SHAPE, "C must be in [1, 2^22), got %lld", (long long)t->C);
    if (t->max_blocks < 1 || t->max_blocks >= ((int64_t)1 << 31) / cache->block_size)
        return fail(FW_E_SHAPE, "need max_blocks >= 1 and max_blocks * block_size < 2^31");
    if (!t->table || !t->lens || !t->free_list || !t->n_free || !t->shared)
        return fail(FW_E_NULL, "cells->table, lens, free_list, n_free and shared are required");
    return FW_OK;
}

fw_status check_fork(const fw_cache *cache, const fw_cells *cells, int64_t P) {
    fw_status s = check_cells(cache, cells);
    if (s != FW_OK) return s;
    if (P < 0 || P >= ((int64_t)1 << 22)) return fail(FW_E_SHAPE, "P must be in [0, 2^22), got %lld", (long long)P);
    return FW_OK;
}

fw_status check_cell_compact(const fw_cache *cache, const fw_cells *cells, int64_t P, int64_t n_kept) {
    fw_status s = check_fork(cache, cells, P);
    if (s != FW_OK) return s;
    // a workgroup of 1024 threads for each listed cell: a grid holds fewer than 2^32 threads
    if (n_kept < 0 || n_kept / 256 + P >= ((int64_t)1 << 22))
        return fail(FW_E_SHAPE, "need n_kept >= 0 and n_kept / 256 + P < 2^22");
    return FW_OK;
}

fw_status check_select(int64_t C, int64_t n, int64_t recent, int64_t n_kept) {
    if (C < 1 || C >= ((int64_t)1 << 22)) return fail(FW_E_SHAPE, "C must be in [1, 2^22), got %lld", (long long)C);
    if (n < 1 || n >= ((int64_t)1 << 31) - 65536) return fail(FW_E_SHAPE, "n must be in [1, 2^31 - 65536)");
    // a grid holds fewer than 2^32 threads: 1024 for a cell, and for 8192 of its tokens where rows are long
    if (C * (n / 8192 + 1) >= ((int64_t)1 << 22)) return fail(FW_E_SHAPE, "C * (n / 8192 + 1) must be < 2^22");
    if (recent < 0) return fail(FW_E_SHAPE, "recent must be >= 0");
    if (n_kept < 0 || n_kept >= ((int64_t)1 << 40)) return fail(FW_E_SHAPE, "n_kept must be in [0, 2^40)");
    return FW_OK;
}

}  // namespace

extern "C" {

size_t fw_prompt_attention_workspace_size(const fw_packed *packed) {
    if (check_packed(packed) != FW_OK) return 0;
    return prompt_layout(*packed, nullptr).bytes;
}

fw_status fw_prompt_attention(const fw_packed *packed, void *o, float *lse, void *ws, size_t ws_bytes,
                              fw_stream stream) {
    fw_status s = check_packed(packed);
    if (s != FW_OK) return s;
    if (packed->Tq == 0) return FW_OK;
    if (!o) return fail(FW_E_NULL, "o is required");
    const PromptWs w = prompt_layout(*packed, ws);
    if ((s = check_ws(ws, ws_bytes, w.bytes)) != FW_OK) return s;
    return hip_status(fw::launch_prompt(*packed, o, lse, w.splits, w.part_o, w.part_lse, (hipStream_t)stream),
                      "fw_prompt_attention");
}

// ---------------------------------------------------------------------------
size_t fw_block_tables_workspace_size(int64_t C) {
    if (C < 1 || C >= ((int64_t)1 << 24)) return 0;
    return fw::tables_ws_bytes(C);
}

fw_status fw_block_tables(int64_t C, const int32_t *old_len, const int32_t *new_len, int32_t block_size,
                          int64_t max_blocks, int32_t *table, int64_t n_blocks, int32_t *free_list, int32_t *n_free,
                          int64_t n_slots, int64_t *slots, int64_t *offsets, int32_t *lens, int32_t *refused, void *ws,
                          size_t ws_bytes, fw_stream stream) {
    constexpr int64_t m31 = (int64_t)1 << 31;
    if (C < 1 || C >= ((int64_t)1 << 24)) return fail(FW_E_SHAPE, "C must be in [1, 2^24), got %lld", (long long)C);
    fw_status s = check_block(block_size);
    if (s != FW_OK) return s;
    if (max_blocks < 1 || max_blocks >= m31 / block_size)
        return fail(FW_E_SHAPE, "need max_blocks >= 1 and max_blocks * block_size < 2^31");
    if (n_blocks < 1 || n_blocks >= m31) return fail(FW_E_SHAPE, "n_blocks must be in [1, 2^31)");
    if (n_slots < 0 || n_slots >= ((int64_t)1 << 40)) return fail(FW_E_SHAPE, "n_slots must be in [0, 2^40)");
    if (!old_len || !new_len || !table || !free_list || !n_free || !offsets || !lens || !refused)
        return fail(FW_E_NULL, "old_len, new_len, table, free_list, n_free, offsets, lens and refused are required");
    if (n_slots > 0 && !slots) return fail(FW_E_NULL, "slots is NULL");
    if ((s = check_ws(ws, ws_bytes, fw::tables_ws_bytes(C))) != FW_OK) return s;
    return hip_status(fw::launch_tables(C, old_len, new_len, block_size, max_blocks, table, n_blocks, free_list, n_free,
                                        n_slots, slots, offsets, lens, refused, ws, (hipStream_t)stream),
                      "fw_block_tables");
}

// ---------------------------------------------------------------------------
int32_t fw_cache_row(int64_t d) { return fw::cache_row(d); }

size_t fw_cache_store_workspace_size(const fw_cache *cache, int64_t N) {
    (void)cache;
    (void)N;
    return 0;
}

fw_status fw_cache_store(const fw_cache *cache, int32_t dtype, const void *k, int64_t k_row, const void *v,
                         int64_t v_row, int64_t N, const int64_t *slots, void *ws, size_t ws_bytes, fw_stream stream) {
    (void)ws;
    (void)ws_bytes;
    fw_status s = check_cache(cache);
    if (s != FW_OK) return s;
    if (dtype != FW_F32 && dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)dtype);
    // a grid holds fewer than 2^32 threads: 256 for 16 rows or more
    if (N < 0 || N > ((int64_t)1 << 28) - 16) return fail(FW_E_SHAPE, "N must be in [0, 2^28 - 16]");
    if (k_row < 0 || v_row < 0 || k_row >= ((int64_t)1 << 31) || v_row >= ((int64_t)1 << 31))
        return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (N == 0) return FW_OK;
    if (!k || !v || !slots) return fail(FW_E_NULL, "k, v and slots are required");
    return hip_status(fw::launch_store(*cache, dtype, k, k_row, v, v_row, N, slots, (hipStream_t)stream),
                      "fw_cache_store");
}

// ---------------------------------------------------------------------------
size_t fw_cache_attention_workspace_size(const fw_cache *cache, int64_t S, int64_t T, int64_t Hq, int64_t Hkv,
                                         int64_t max_blocks) {
    if (check_cache(cache) != FW_OK || check_decode(cache->block_size, S, T, Hq, Hkv, max_blocks) != FW_OK) return 0;
    return fw::decode_ws_bytes(S * Hkv, T * (Hq / Hkv), cache->d, max_blocks, cache->block_size);
}

fw_status fw_cache_attention(const fw_cache *cache, int32_t dtype, const void *q, int64_t S, int64_t T, int64_t Hq,
                             int64_t Hkv, int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table,
                             int64_t max_blocks, const int32_t *lens, const float *scale, void *o, float *lse, void *ws,
                             size_t ws_bytes, fw_stream stream) {
    fw_status s = check_cache(cache);
    if (s != FW_OK) return s;
    if (dtype != FW_F32 && dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)dtype);
    if ((s = check_decode(cache->block_size, S, T, Hq, Hkv, max_blocks)) != FW_OK) return s;
    constexpr int64_t m31 = (int64_t)1 << 31;
    if (q_seq < 0 || q_tok < 0 || q_head < 0 || q_seq >= m31 || q_tok >= m31 || q_head >= m31)
        return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (!q || !table || !lens || !o) return fail(FW_E_NULL, "q, table, lens and o are required");
    if ((s = check_ws(ws, ws_bytes,
                      fw::decode_ws_bytes(S * Hkv, T * (Hq / Hkv), cache->d, max_blocks, cache->block_size))) != FW_OK)
        return s;
    return hip_status(fw::launch_decode(*cache, dtype, q, S, T, Hq, Hkv, q_seq, q_tok, q_head, table, max_blocks, lens,
                                        scale, o, lse, ws, (hipStream_t)stream),
                      "fw_cache_attention");
}

// ---------------------------------------------------------------------------
size_t fw_rotate_heads_workspace_size(const fw_heads *heads) {
    (void)heads;
    return 0;
}

fw_status fw_rotate_heads(const fw_heads *heads, void *q_out, int64_t qo_row, int64_t qo_head, void *k_out,
                          int64_t ko_row, int64_t ko_head, void *ws, size_t ws_bytes, fw_stream stream) {
    (void)ws;
    (void)ws_bytes;
    fw_status s = check_heads(heads);
    if (s != FW_OK) return s;
    constexpr int64_t m31 = (int64_t)1 << 31;
    const int64_t strides[] = {qo_row, qo_head, ko_row, ko_head};
    for (int64_t x : strides)
        if (x < 0 || x >= m31) return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (!rows_apart(heads->T, heads->Hq, heads->d, qo_row, qo_head) || !rows_apart(heads->T, heads->Hkv, heads->d, ko_row, ko_head))
        return fail(FW_E_SHAPE, "rows of an output meet each other");
    if (heads->T == 0 || heads->Hq + heads->Hkv == 0) return FW_OK;
    if ((heads->Hq > 0 && !q_out) || (heads->Hkv > 0 && !k_out)) return fail(FW_E_NULL, "q_out or k_out is NULL");
    if ((heads->Hq > 0 && q_out == heads->q && (qo_row != heads->q_row || qo_head != heads->q_head)) ||
        (heads->Hkv > 0 && k_out == heads->k && (ko_row != heads->k_row || ko_head != heads->k_head)))
        return fail(FW_E_SHAPE, "an output in its input's place needs its strides");
    return hip_status(fw::launch_rotate(*heads, q_out, qo_row, qo_head, k_out, ko_row, ko_head, (hipStream_t)stream),
                      "fw_rotate_heads");
}

// ---------------------------------------------------------------------------
size_t fw_cache_scores_workspace_size(const fw_cache *cache, int64_t S, int64_t T, int64_t Hq, int64_t Hkv,
                                      int64_t max_blocks) {
    (void)cache;
    (void)S;
    (void)T;
    (void)Hq;
    (void)Hkv;
    (void)max_blocks;
    return 0;
}

fw_status fw_cache_scores(const fw_cache *cache, int32_t dtype, const void *q, int64_t S, int64_t T, int64_t Hq,
                          int64_t Hkv, int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table,
                          int64_t max_blocks, const int32_t *lens, const float *scale, const float *lse,
                          const float *earlier, float *scores, int64_t n, void *ws, size_t ws_bytes, fw_stream stream) {
    (void)ws;
    (void)ws_bytes;
    fw_status s = check_cache(cache);
    if (s != FW_OK) return s;
    if (dtype != FW_F32 && dtype != FW_BF16) return fail(FW_E_DTYPE, "unknown dtype %d", (int)dtype);
    if ((s = check_decode(cache->block_size, S, T, Hq, Hkv, max_blocks)) != FW_OK) return s;
    constexpr int64_t m31 = (int64_t)1 << 31;
    if (q_seq < 0 || q_tok < 0 || q_head < 0 || q_seq >= m31 || q_tok >= m31 || q_head >= m31)
        return fail(FW_E_SHAPE, "strides must be in [0, 2^31)");
    if (n < 1 || n >= m31) return fail(FW_E_SHAPE, "n must be in [1, 2^31)");
    if (!q || !table || !lens || !lse || !scores) return fail(FW_E_NULL, "q, table, lens, lse and scores are required");
    return hip_status(fw::launch_cache_scores(*cache, dtype, q, S, T, Hq, Hkv, q_seq, q_tok, q_head, table, max_blocks,
                                              lens, scale, lse, earlier, scores, n, (hipStream_t)stream),
                      "fw_cache_scores");
}

// ---------------------------------------------------------------------------
size_t fw_cache_select_workspace_size(int64_t C, int64_t n) {
    if (check_select(C, n, 0, 0) != FW_OK) return 0;
    return fw::select_ws_bytes(C, n);
}

fw_status fw_cache_select(int64_t C, const float *scores, int64_t n, const int32_t *lens, const int32_t *keep,
                          int64_t recent, int64_t n_kept, int64_t *offsets, int32_t *kept_pos, void *ws,
                          size_t ws_bytes, fw_stream stream) {
    fw_status s = check_select(C, n, recent, n_kept);
    if (s != FW_OK) return s;
    if (!scores || !lens || !keep || !offsets) return fail(FW_E_NULL, "scores, lens, keep and offsets are required");
    if (n_kept > 0 && !kept_pos) return fail(FW_E_NULL, "kept_pos is NULL");
    if ((s = check_ws(ws, ws_bytes, fw::select_ws_bytes(C, n))) != FW_OK) return s;
    return hip_status(fw::launch_select_cells(C, scores, n, lens, keep, recent, n_kept, offsets, kept_pos, ws,
                                              (hipStream_t)stream),
                      "fw_cache_select");
}

// ---------------------------------------------------------------------------
size_t fw_cache_fork_workspace_size(const fw_cache *cache, const fw_cells *cells, int64_t P) {
    if (check_fork(cache, cells, P) != FW_OK) return 0;
    return fw::pages_ws_bytes(*cache, *cells, 1, P, 0);
}

fw_status fw_cache_fork(const fw_cache *cache, const fw_cells *cells, int64_t P, const int32_t *src,
                        const int32_t *dst, const int32_t *length, int32_t *refused, void *ws, size_t ws_bytes,
                        fw_stream stream) {
    fw_status s = check_fork(cache, cells, P);
    if (s != FW_OK) return s;
    if (!refused || (P > 0 && (!src || !dst))) return fail(FW_E_NULL, "src, dst and refused are required");
    if ((s = check_ws(ws, ws_bytes, fw::pages_ws_bytes(*cache, *cells, 1, P, 0))) != FW_OK) return s;
    return hip_status(fw::launch_fork(*cache, *cells, P, src, dst, length, refused, ws, (hipStream_t)stream),
                      "fw_cache_fork");
}

size_t fw_cache_release_workspace_size(const fw_cache *cache, const fw_cells *cells) {
    if (check_cells(cache, cells) != FW_OK) return 0;
    return fw::pages_ws_bytes(*cache, *cells, 0, 0, 0);
}

fw_status fw_cache_release(const fw_cache *cache, const fw_cells *cells, const int32_t *new_len, int32_t *refused,
                           void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status s = check_cells(cache, cells);
    if (s != FW_OK) return s;
    if (!new_len || !refused) return fail(FW_E_NULL, "new_len and refused are required");
    if ((s = check_ws(ws, ws_bytes, fw::pages_ws_bytes(*cache, *cells, 0, 0, 0))) != FW_OK) return s;
    return hip_status(fw::launch_release(*cache, *cells, new_len, refused, ws, (hipStream_t)stream), "fw_cache_release");
}

size_t fw_cache_compact_workspace_size(const fw_cache *cache, const fw_cells *cells, int64_t P, int64_t n_kept) {
    if (check_cell_compact(cache, cells, P, n_kept) != FW_OK) return 0;
    return fw::pages_ws_bytes(*cache, *cells, 2, P, n_kept);
}

fw_status fw_cache_compact(const fw_cache *cache, const fw_cells *cells, int64_t P, const int32_t *which,
                           const int64_t *offsets, int64_t n_kept, const int32_t *kept_pos, int32_t *refused,
                           void *ws, size_t ws_bytes, fw_stream stream) {
    fw_status s = check_cell_compact(cache, cells, P, n_kept);
    if (s != FW_OK) return s;
    if (!which && P > cells->C) return fail(FW_E_SHAPE, "P = %lld cells of %lld", (long long)P, (long long)cells->C);
    if (!refused || (P > 0 && !offsets)) return fail(FW_E_NULL, "offsets and refused are required");
    if (n_kept > 0 && !kept_pos) return fail(FW_E_NULL, "kept_pos is NULL");
    if ((s = check_ws(ws, ws_bytes, fw::pages_ws_bytes(*cache, *cells, 2, P, n_kept))) != FW_OK) return s;
    return hip_status(fw::launch_cell_compact(*cache, *cells, P, which, offsets, n_kept, kept_pos, refused, ws,
                                              (hipStream_t)stream),
                      "fw_cache_compact");
}

}  // extern "C"
