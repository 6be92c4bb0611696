// Internal launch interface between the C ABI layer and the kernels.
#pragma once

#include "fw_common.hpp"

namespace fw {

// Budgets of one fw_dense_topk call, sorted ascending; perm[t] is the
// caller's position of the t-th smallest budget.
struct KsArg {
    int n;
    int k[FW_MAX_KS];
    int perm[FW_MAX_KS];
};

// k_topk.hip
hipError_t launch_scores(int dtype, const void *q, const void *k, const float *scale,
                         const float *bias, int64_t H, int64_t G, int64_t n, int d, float *z,
                         hipStream_t st);
hipError_t launch_select(const float *z, int64_t R, int64_t n, const KsArg &ks, float *row_m,
                         float *row_l, uint32_t *thr_key, int32_t *thr_cut, int32_t *topk_idx,
                         int kmax, hipStream_t st);
// key ranges that launch_tiers' sums are split into; with more than one it
// takes part [splits][R][n_ks + 1][d] and part_m [splits][R][n_ks + 1]
int tiers_splits(int dtype, int64_t H, int64_t G, int64_t n);
hipError_t launch_tiers(int dtype, const void *v, const float *z, const float *row_m, const float *row_l,
                        const uint32_t *thr_key, const int32_t *thr_cut, int64_t H, int64_t G, int64_t n, int d,
                        const KsArg &ks, float *o, float *o_s, float *gap, float *dropped, int splits, float *part,
                        float *part_m, hipStream_t st);

// k_topk_fused.hip -- one-kernel path for bf16, d = 128, n in {1024, 2048, 4096}
bool fused_topk_supported(const fw_rows &rows, const KsArg &ks);
size_t fused_topk_ws_bytes(const fw_rows &rows, int kmax);
hipError_t launch_fused_topk(const fw_rows &rows, const KsArg &ks, float *o, float *o_s, float *gap,
                             float *dropped, int32_t *topk_idx, void *ws, hipStream_t st);

// k_topk_mp.hip -- multi-pass one-kernel path for bf16, d = 128, n a multiple
// of 32 up to 4096, 128 rows per unit tile (same workspace as the fused path)
bool mp_topk_supported(const fw_rows &rows, const KsArg &ks);
hipError_t launch_mp_topk(const fw_rows &rows, const KsArg &ks, float *o, float *o_s, float *gap,
                          float *dropped, int32_t *topk_idx, void *ws, hipStream_t st);

// k_subset.hip -- exhaustive best subset (float64)
size_t best_subset_ws_bytes(int64_t n, int k);
bool best_subset_plannable(int64_t n, int k);
hipError_t launch_best_subset(const fw_rows &rows, int k, int32_t *best_idx, float *best_gap,
                              float *topk_gap, float *closed, float *dropped_topk,
                              int32_t *topk_idx, void *ws, hipStream_t st);

// k_pool.hip -- candidate-set search (ES_pool, pool balancing, certificate)
bool pool_plannable(int64_t N, int d, int nb, const int32_t *s, const int32_t *extra);
size_t pool_ws_bytes(const fw_rows &rows, int nb, const int32_t *s, const int32_t *extra);
hipError_t launch_pool(const fw_rows &rows, int nb, const int32_t *s, const int32_t *extra, int max_swaps,
                       int fw_iters, int32_t *pool_idx, int32_t *best_idx, int32_t *bal_idx, int32_t *geo_idx,
                       int32_t *n_swaps, float *stats,
                       float flat_threshold, float *cell_median, uint8_t *cell_flat, void *ws, hipStream_t st);

// k_vote.hip -- group vote
bool vote_supported(const fw_rows &rows, int s, int gs);
hipError_t launch_vote(const fw_rows &rows, int s, int gs, int32_t *vote_idx, float *es_vote, float *es_top,
                       float *dropped, hipStream_t st);

// k_swap.hip -- swap rule
size_t swap_ws_bytes(const fw_rows &rows, int k, int max_iters);
hipError_t launch_swap(const fw_rows &rows, int k, int max_iters, int32_t *s_idx, float *gap_traj,
                       int32_t *n_swaps, float *dropped, void *ws, hipStream_t st);

// k_curve.hip -- window importance and dropped-mass curve
size_t curve_ws_bytes(const fw_rows &rows);
hipError_t launch_curve(const fw_rows &rows, float *importance, float *curve, int32_t *order,
                        void *ws, hipStream_t st);

// k_window.hip -- window importance on MFMA (bf16, d = 128, 16..64 rows)
bool window_mfma_supported(const fw_rows &rows);
void launch_window_mfma(const fw_rows &rows, float *part_m, float *part_l, float *row_m, float *row_il,
                        float *importance, hipStream_t st);

// k_compact.hip -- global allocation and ragged compaction
size_t compact_ws_bytes(int64_t H, int64_t n);
hipError_t launch_compact(int dtype, const void *k, const void *v, int64_t H, int64_t hpl,
                          int64_t n, int64_t d, const float *importance, int64_t budget,
                          int floor, int64_t cap, int64_t *offsets, int32_t *kept_pos, void *k_out,
                          void *v_out, float *tau, float *dropped, int64_t *bytes_held, void *ws,
                          hipStream_t st);
hipError_t launch_maxpool(const float *scores, int64_t H, int64_t n, int kernel, float *out, hipStream_t st);


// k_prompt.hip -- attention of packed prompts; with more than one split it
// takes part_o [splits][Tq][Hq][d] and part_lse [splits][Tq][Hq]
int prompt_splits(const fw_packed &p);
hipError_t launch_prompt(const fw_packed &p, void *o, float *lse, int splits, float *part_o, float *part_lse,
                         hipStream_t st);

// bytes of a cached key's row (fw_cache_row)
inline int cache_row(int64_t d) {
    constexpr int rows[] = {32, 64, 96, 128, 192, 256};
    if (d < 1) return 0;
    for (int r : rows)
        if (d <= r) return r;
    return 0;
}

// k_cache.hip -- block tables and the 8-bit cache's store
size_t tables_ws_bytes(int64_t C);
hipError_t launch_tables(int64_t C, const int32_t *old_len, const int32_t *new_len, int block_size, int64_t W,
                         int32_t *table, int64_t n_blocks, int32_t *free_list, int32_t *n_free, int64_t n_slots,
                         int64_t *slots, int64_t *offsets, int32_t *lens, int32_t *refused, void *ws, hipStream_t st);
hipError_t launch_store(const fw_cache &cache, int dtype, const void *k, int64_t k_row, const void *v, int64_t v_row,
                        int64_t N, const int64_t *slots, hipStream_t st);

// k_decode.hip -- attention over the 8-bit cache
size_t decode_ws_bytes(int64_t C, int64_t R, int64_t d, int64_t W, int block_size);
hipError_t launch_decode(const fw_cache &cache, int dtype, const void *q, int64_t S, int64_t T, int64_t Hq, int64_t Hkv,
                         int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table, int64_t W,
                         const int32_t *lens, const float *scale, void *o, float *lse, void *ws, hipStream_t st);

// k_rotate.hip -- norm and rotation of queries and keys
hipError_t launch_rotate(const fw_heads &heads, void *q_out, int64_t qo_row, int64_t qo_head, void *k_out, int64_t ko_row,
                         int64_t ko_head, hipStream_t st);

// k_scores.hip -- scores of cached tokens and the choice among them
hipError_t launch_cache_scores(const fw_cache &cache, int dtype, const void *q, int64_t S, int64_t T, int64_t Hq,
                               int64_t Hkv, int64_t q_seq, int64_t q_tok, int64_t q_head, const int32_t *table,
                               int64_t W, const int32_t *lens, const float *scale, const float *lse,
                               const float *earlier, float *scores, int64_t n, hipStream_t st);
hipError_t launch_select_cells(int64_t C, const float *scores, int64_t n, const int32_t *lens, const int32_t *keep,
                               int64_t recent, int64_t n_kept, int64_t *offsets, int32_t *kept_pos, void *ws,
                               hipStream_t st);
size_t select_ws_bytes(int64_t C, int64_t n);

// k_pages.hip -- cells that share blocks (kind 0: release, 1: fork of P pairs, 2: compaction of P cells)
size_t pages_ws_bytes(const fw_cache &cache, const fw_cells &cells, int kind, int64_t P, int64_t n_kept);
hipError_t launch_release(const fw_cache &cache, const fw_cells &cells, const int32_t *new_len, int32_t *refused,
                          void *ws, hipStream_t st);
hipError_t launch_fork(const fw_cache &cache, const fw_cells &cells, int64_t P, const int32_t *src, const int32_t *dst,
                       const int32_t *length, int32_t *refused, void *ws, hipStream_t st);
hipError_t launch_cell_compact(const fw_cache &cache, const fw_cells &cells, int64_t P, const int32_t *which,
                               const int64_t *offsets, int64_t n_kept, const int32_t *kept_pos, int32_t *refused,
                               void *ws, hipStream_t st);

}  // namespace fw
