// Internal launch interface of the operators of a layer held in 4 bits (mc_layer_q4_*).
#pragma once
#include "mc_common.cuh"

namespace mc {

constexpr int kQ4MaxSelectLen = 1 << 19;  // longest sequence mc_layer_q4_select takes: a key per page in shared memory

// Rows of the append and read calls, in the caller's arrays.
struct Q4RowArgs {
  const int32_t* begin;  // read: [batch] or null
  const int32_t* row_offsets;
  int n_rows;
  long long k_stride, v_stride;  // elements
};
mc_status launch_layer_q4_append(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer, const void* k,
                                 const void* v, const Q4RowArgs& rows, cudaStream_t stream);
mc_status launch_layer_q4_read(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer, void* k, void* v,
                               const Q4RowArgs& rows, cudaStream_t stream);

size_t layer_q4_select_workspace_bytes(const mc_config* cfg, const mc_batch* bt);
mc_status launch_layer_q4_select(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer,
                                 const mc_score_opts* opts, const mc_page_selection* keep, const void* q, int32_t* pages, int32_t* counts,
                                 void* workspace, cudaStream_t stream);

size_t layer_q4_attn_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int flags);
mc_status launch_layer_q4_attn(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer,
                               const mc_score_opts* opts, const int32_t* pages, const int32_t* counts, int pages_stride, const void* q,
                               const void* k_new, const void* v_new, int flags, void* out, float* lse, void* workspace,
                               cudaStream_t stream);

}  // namespace mc
