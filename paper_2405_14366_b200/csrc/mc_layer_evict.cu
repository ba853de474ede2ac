// Eviction from one uncompressed layer's cache by accumulated attention weight: per (sequence, kv head) the `budget`
// rows with the largest key stay (guarded rows -- the first positions and the most recent ones -- before all others,
// then by weight, ties to the lower index).  Rows that stay inside the first `budget` slots are not touched; the k-th
// row that stays behind them moves into the k-th slot that fell free before them.  So one decode step that evicts one
// token moves one row, and nothing is read that is also written: sources lie at or behind `budget`, targets before it.
//
// A cluster of CTAs per segment: every CTA keeps the ordered 32-bit keys of its share of the tokens in shared memory,
// the budget-th largest key is found digit by digit (11 + 11 + 10 bits: a histogram per CTA, summed over the
// cluster through distributed shared memory), then holes and movers are listed in index order (a warp per run of
// tokens, counts scanned over the cluster) and the cluster's warps copy the rows.  Bytes: 8 per token for the
// keys, 2 x 512 per moved row; short caches are bound by the chain of barriers (about a microsecond per digit).
#include <cooperative_groups.h>

#include <algorithm>

#include "mc_layer.cuh"
#include "mc_layer.h"
#include "mc_kernels.h"

namespace mc {
namespace cg = cooperative_groups;

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBins = 2048;
constexpr int kEvMaxCluster = 8;
constexpr int kEvSmemKeys = 40 * 1024;  // keys of a CTA's share held in shared memory (160 KB); a longer share is read again

struct EvictParams {
  Geom g;
  char* k_pool;
  char* v_pool;
  int32_t* positions;
  float* weights;
  int32_t* status;
  const int32_t* q_pos;
  int32_t* new_lens;
  int32_t* lists;  // [segment][holes, movers][list_stride]
  int list_stride;
  int budget, n_sink, n_recent;
  int smem_keys;  // keys this launch has shared memory for, per CTA
};

// Order-preserving 32-bit key of a weight: larger weight, larger key; NaN lowest, -0 = +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Exclusive sum over the block of one int per warp (lane 0's), for every warp, and the total.
__device__ __forceinline__ int warp_prefix(int v, int* s, int warp, int lane, int& total) {
  __syncthreads();
  if (lane == 0) s[warp] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kEvWarps; ++k) {
    const int x = s[k];
    if (k < warp) before += x;
    all += x;
  }
  total = all;
  return before;
}

__global__ void __launch_bounds__(kEvThreads) layer_evict_kernel(const __grid_constant__ EvictParams p) {
  // (no early start of the kernel behind: it may take new_lens for its lengths, which are read before the wait)
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  extern __shared__ uint32_t smem_u[];
  uint32_t* hist = smem_u;                            // [3][kEvBins]
  uint32_t* keys = hist + 3 * kEvBins;                // [smem_keys]
  uint32_t* mask = keys + p.smem_keys;                // [(smem_keys + 31) / 32 + 1]: who stays, a bit per token
  __shared__ int warp_s[kEvWarps];
  __shared__ int pub[4];                              // read by the cluster: ties, holes, movers of this CTA
  __shared__ int found[2];                            // digit, how many keys lie above it
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads, ps = p.g.page_size, shift = p.g.page_shift;
  const int seg = blockIdx.x / C, b = seg / H, head = seg - b * H;
  grid_dep_wait();
  const int raw = p.g.seq_lens[b];
  const int n = min(max(raw, 0), p.g.max_seq_len);
  if (head == 0 && rank == 0 && tid == 0) {
    if (raw != n) atomicOr(p.status, MC_FLAG_BAD_METADATA);
    p.new_lens[b] = min(n, p.budget);
  }
  if (n <= p.budget) return;  // (the whole cluster)
  const int last = max(p.q_pos ? p.q_pos[b] : n - 1, -1);
  const int recent = last - p.n_recent;  // positions above it are guarded
  const int per = (n + C - 1) / C;
  const int i0 = min(n, rank * per), cnt = min(n, i0 + per) - i0;  // this CTA's tokens
  const int32_t* table = p.g.block_table + (size_t)b * p.g.max_pages_per_seq;
  const bool held = per <= p.smem_keys;

  auto slot_of = [&](int t) -> long long {  // slot of the [page][head][row] pools; -1: not a page
    const int page = table[t >> shift];
    if (!page_ok(p.g, page)) return -1;
    return ((long long)page * H + head) * ps + (t & (ps - 1));
  };
  auto load_key = [&](int i) -> uint32_t {
    const long long at = slot_of(i0 + i);
    if (at < 0) {
      atomicOr(p.status, MC_FLAG_BAD_METADATA);
      return 0u;
    }
    const int pos = p.positions[at];
    const float w = p.weights[at];
    return (pos < p.n_sink || pos > recent) ? 0xffffffffu : weight_key(w);
  };
  auto key_at = [&](int i) -> uint32_t { return held ? keys[i] : load_key(i); };

  for (int i = tid; i < 3 * kEvBins; i += kEvThreads) hist[i] = 0;
  __syncthreads();
  // ---- the budget-th largest key ------------------------------------------------------------------
  uint32_t prefix = 0;       // digits found so far
  int want = p.budget;       // rank of the key among those that share the prefix
#pragma unroll
  for (int d = 0; d < 3; ++d) {
    const int sh = d == 0 ? 21 : (d == 1 ? 10 : 0), bits = d == 2 ? 10 : 11;
    uint32_t* h = hist + d * kEvBins;
    for (int i = tid; i < cnt; i += kEvThreads) {
      uint32_t k;
      if (d == 0 || !held) {
        k = load_key(i);
        if (d == 0 && held) keys[i] = k;
      } else {
        k = keys[i];
      }
      if (d == 0 || (k >> (sh + bits)) == prefix) atomicAdd(&h[(k >> sh) & ((1u << bits) - 1)], 1u);
    }
    cl.sync();
    // every CTA sums the cluster's histograms for itself: a thread takes four digits, the largest first
    int c4[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int bin = kEvBins - 1 - (4 * tid + k);
      int v = 0;
      for (int r = 0; r < C; ++r) v += (int)cl.map_shared_rank(h, r)[bin];
      c4[k] = v;
      sum += v;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    int total;
    const int before = warp_prefix(__shfl_sync(0xffffffffu, incl, 31), warp_s, warp, lane, total);
    int above = before + incl - sum;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (above < want && want <= above + c4[k]) {
        found[0] = kEvBins - 1 - (4 * tid + k);
        found[1] = above;
      }
      above += c4[k];
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)found[0];
    want -= found[1];
  }
  // all keys above `prefix` stay, and the first `want` of those equal to it.  A warp owns a run of tokens.
  const uint32_t thr = prefix;
  const int words = (cnt + 31) / 32, wper = (words + kEvWarps - 1) / kEvWarps;
  const int w0 = min(words, warp * wper), w1 = min(words, w0 + wper);
  int ties = 0;
  for (int w = w0; w < w1; ++w) {
    const int i = 32 * w + lane;
    ties += __popc(__ballot_sync(0xffffffffu, i < cnt && key_at(i) == thr));
  }
  int total_ties;
  int tie = warp_prefix(ties, warp_s, warp, lane, total_ties);
  if (tid == 0) pub[0] = total_ties;
  cl.sync();
  for (int r = 0; r < rank; ++r) tie += *cl.map_shared_rank(&pub[0], r);
  // ---- who stays; holes before the budget, movers behind it ------------------------------------------
  auto stay_word = [&](int w, int& t) -> uint32_t {
    const int i = 32 * w + lane;
    const uint32_t k = i < cnt ? key_at(i) : 0u;
    const uint32_t eq = __ballot_sync(0xffffffffu, i < cnt && k == thr);
    const bool stay = i < cnt && (k > thr || (k == thr && t + __popc(eq & ((1u << lane) - 1u)) < want));
    t += __popc(eq);
    return __ballot_sync(0xffffffffu, stay);
  };
  int holes = 0, movers = 0, tie_w = tie;
  for (int w = w0; w < w1; ++w) {
    const uint32_t s = stay_word(w, tie_w);
    if (held && lane == 0) mask[w] = s;
    const int rel = p.budget - (i0 + 32 * w);  // tokens of this word before the budget
    const uint32_t low = rel >= 32 ? 0xffffffffu : (rel <= 0 ? 0u : (1u << rel) - 1u);
    const int valid = cnt - 32 * w;
    const uint32_t here = valid >= 32 ? 0xffffffffu : (1u << valid) - 1u;
    holes += __popc(~s & low & here);
    movers += __popc(s & ~low);
  }
  int total_h, total_m;
  int at_h = warp_prefix(holes, warp_s, warp, lane, total_h);
  int at_m = warp_prefix(movers, warp_s, warp, lane, total_m);
  if (tid == 0) {
    pub[1] = total_h;
    pub[2] = total_m;
  }
  cl.sync();
  int n_moves = 0;
  for (int r = 0; r < C; ++r) {
    const int* q = cl.map_shared_rank(&pub[0], r);
    const int m = q[2];
    if (r < rank) {
      at_h += q[1];
      at_m += m;
    }
    n_moves += m;
  }
  int32_t* hole_l = p.lists + (size_t)seg * 2 * p.list_stride;
  int32_t* move_l = hole_l + p.list_stride;
  for (int w = w0; w < w1; ++w) {
    const uint32_t s = held ? mask[w] : stay_word(w, tie);
    const int i = 32 * w + lane, t = i0 + i;
    const bool stay = (s >> lane) & 1u;
    const bool hole = i < cnt && t < p.budget && !stay, mover = stay && t >= p.budget;
    const uint32_t hb = __ballot_sync(0xffffffffu, hole), mb = __ballot_sync(0xffffffffu, mover), lt = (1u << lane) - 1u;
    if (hole) hole_l[at_h + __popc(hb & lt)] = t;
    if (mover) move_l[at_m + __popc(mb & lt)] = t;
    at_h += __popc(hb);
    at_m += __popc(mb);
  }
  cl.sync();  // the lists are complete (and nobody reads another CTA's shared memory from here on)
  // ---- the rows: a lane works a move's slots out, then the warp copies it (lanes 0..15 K, 16..31 V) -------
  const int n_warps = C * kEvWarps, gw = rank * kEvWarps + warp;
  const int share = min(32, max(1, (n_moves + n_warps - 1) / n_warps));
  char* pool = lane < 16 ? p.k_pool : p.v_pool;
  for (int m0 = gw * share; m0 < n_moves; m0 += n_warps * share) {
    const int m = m0 + lane;
    long long src = -1, dst = -1;
    if (lane < share && m < n_moves) {
      src = slot_of(__ldcg(move_l + m));
      dst = slot_of(__ldcg(hole_l + m));
      if (src >= 0 && dst >= 0) {
        p.weights[dst] = p.weights[src];
        p.positions[dst] = p.positions[src];
      }
    }
    const int live = min(share, n_moves - m0);
    for (int k0 = 0; k0 < live; k0 += 4) {  // four rows in flight
      uint4 v[4];
      long long to[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long from = __shfl_sync(0xffffffffu, src, (k0 + k) & 31);
        to[k] = __shfl_sync(0xffffffffu, dst, (k0 + k) & 31);
        if (k0 + k >= live || from < 0) to[k] = -1;
        if (to[k] >= 0) v[k] = ld_stream16(pool + from * kRowBytes + (lane & 15) * 16);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (to[k] >= 0) st_stream16(pool + to[k] * kRowBytes + (lane & 15) * 16, v[k]);
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------
static int evict_list_stride(const mc_batch* bt) { return (bt->max_seq_len + 1) / 2 + 1; }  // min(budget, n - budget) at most
size_t layer_evict_workspace_bytes(const mc_config* cfg, const mc_batch* bt) {
  return align_up((size_t)bt->batch * cfg->n_kv_heads * 2 * evict_list_stride(bt) * 4, 256);
}

mc_status launch_layer_evict(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                             const mc_evict_opts* opts, int32_t* new_lens, void* workspace, cudaStream_t stream) {
  if (bt->batch == 0) return MC_OK;
  EvictParams ep;
  ep.g = g;
  ep.k_pool = (char*)layer->k_pool;
  ep.v_pool = (char*)layer->v_pool;
  ep.positions = layer->positions;
  ep.weights = layer->weights;
  ep.status = layer->status;
  ep.q_pos = opts->q_pos;
  ep.new_lens = new_lens;
  ep.lists = (int32_t*)workspace;
  ep.list_stride = evict_list_stride(bt);
  ep.budget = opts->budget;
  ep.n_sink = opts->n_sink;
  ep.n_recent = opts->n_recent;
  int cluster = 1;  // about 2048 tokens per CTA
  while (cluster < kEvMaxCluster && bt->max_seq_len > 2048 * cluster) cluster *= 2;
  const int per = (bt->max_seq_len + cluster - 1) / cluster;
  ep.smem_keys = std::min((per + 31) / 32 * 32, kEvSmemKeys);
  const size_t smem = (size_t)(3 * kEvBins + ep.smem_keys + ep.smem_keys / 32 + 1) * 4;
  MC_CUDA_CHECK(cudaFuncSetAttribute(layer_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  cudaLaunchConfig_t cfgl = {};
  cfgl.gridDim = dim3((unsigned)(bt->batch * cfg->n_kv_heads * cluster));
  cfgl.blockDim = dim3(kEvThreads);
  cfgl.dynamicSmemBytes = smem;
  cfgl.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfgl.attrs = attr;
  cfgl.numAttrs = 2;
  MC_CUDA_CHECK(cudaLaunchKernelEx(&cfgl, layer_evict_kernel, ep));
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
