// Internal launch interface of the operators of an uncompressed layer's cache (mc_layer_*).
#pragma once
#include "mc_common.cuh"

namespace mc {

constexpr int kMaxLayerBatch = 512;  // sequences whose unit prefix lives in shared memory

size_t layer_attn_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int flags);
mc_status launch_layer_attn(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                            const mc_score_opts* opts, const void* q, const void* k_new, const void* v_new, int flags, void* out,
                            float* lse, void* workspace, cudaStream_t stream);

constexpr int kMaxObserveRows = 256;  // observed queries x query heads per kv head
size_t layer_observe_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int n_obs);
mc_status launch_layer_observe(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                               const mc_score_opts* opts, const void* q, int n_obs, int flags, void* workspace, cudaStream_t stream);

size_t layer_evict_workspace_bytes(const mc_config* cfg, const mc_batch* bt);
mc_status launch_layer_evict(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                             const mc_evict_opts* opts, int32_t* new_lens, void* workspace, cudaStream_t stream);

}  // namespace mc
