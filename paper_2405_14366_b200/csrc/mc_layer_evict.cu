// Eviction from one uncompressed layer's cache by accumulated attention weight: per (sequence, kv head) the `budget`
// rows with the largest key stay (guarded rows -- the first positions and the most recent ones -- before all others,
// then by weight, ties to the lower index).  Rows that stay inside the first `budget` slots are not touched; the k-th
// row that stays behind them moves into the k-th slot that fell free before them.  So one decode step that evicts one
// token moves one row, and nothing is read that is also written: sources lie at or behind `budget`, targets before it.
//
// A cluster of CTAs per segment (one CTA where the segments alone fill the GPU): every CTA keeps the ordered 32-bit keys
// of its share of the tokens in shared memory, the budget-th largest key is found digit by digit (11 + 11 + 10 bits:
// a histogram per CTA, its non-empty bins added to every CTA's total through distributed shared memory), then holes and
// movers are listed in index order (a warp per run of tokens, counts scanned over the cluster) and the cluster's warps
// copy the rows.  One token too many, the steady state of a bounded cache, needs no digits where a segment has one CTA: the
// smallest key goes (256 segments of 1025 tokens 4.2 us, of 4097 6.8).  Clusters, which few segments of more than 1024
// tokens get, take the general way also then (128 segments of 1025 tokens 13.6 us, 8 of 4097 11.9).
// Bytes: 8 per token for the keys, 2 x 512 per moved row; short caches are bound by the chain of dependent loads and
// barriers.  Measured, from a CUDA graph and with a copy of 2 to 4 us that puts the marks back: 55 us on 8 x 32 segments of
// 4096 tokens down to 1000 (202 MB of rows at 5.6 TB/s in 36 us, the selection before it 12 us), 45 us on 4 x 8 of 32768
// down to 4096 (115 MB in 20 us).
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

// Exclusive sums over the block of two ints per warp, and the totals.
struct Two {
  int a, b;
};
__device__ __forceinline__ Two warp_prefix(Two v, Two* s, int warp, int lane, Two& total) {
  __syncthreads();
  if (lane == 0) s[warp] = v;
  __syncthreads();
  Two before = {0, 0}, all = {0, 0};
#pragma unroll
  for (int k = 0; k < kEvWarps; ++k) {
    const Two x = s[k];
    if (k < warp) {
      before.a += x.a;
      before.b += x.b;
    }
    all.a += x.a;
    all.b += x.b;
  }
  total = all;
  return before;
}

__global__ void __launch_bounds__(kEvThreads, 2) layer_evict_kernel(const __grid_constant__ EvictParams p) {
  // (no early start of the kernel behind: it may take new_lens for its lengths, which are read before the wait)
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  extern __shared__ __align__(16) uint32_t smem_u[];
  uint32_t* total = smem_u;                           // [3][kEvBins]: the cluster's histograms
  uint32_t* local = total + 3 * kEvBins;              // [kEvBins]: this CTA's, digit by digit (clusters only)
  uint32_t* keys = local + kEvBins;                   // [smem_keys]
  uint32_t* mask = keys + p.smem_keys;                // [smem_keys / 32 + 1]: who stays, a bit per token
  __shared__ Two warp_s[kEvWarps];
  __shared__ uint64_t best_s[kEvWarps];
  __shared__ Two pub[kEvMaxCluster], pub_tie[kEvMaxCluster];  // written by the cluster: (holes, movers) and ties of every CTA
  __shared__ int found[3];                            // digit, keys above it, keys equal to it
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads, ps = p.g.page_size, shift = p.g.page_shift;
  const int seg = blockIdx.x / C, b = seg / H, head = seg - b * H;
  grid_dep_wait();
  const int raw = __ldcg(p.g.seq_lens + b);
  const int n = min(max(raw, 0), p.g.max_seq_len);
  const bool scribe = head == 0 && rank == 0 && tid == kEvThreads - 1;
  int was = 0;
  if (scribe) {
    if (raw != n) atomicOr(p.status, MC_FLAG_BAD_METADATA);
    was = atomicExch(p.new_lens + b, min(n, p.budget));
  }
  // The new length is in L2 before this grid ends, since the kernel behind may read it before its wait: an exchange has
  // happened when what was there before is back, and this waits for that.  (8 x 32 segments of 1025 tokens, marks put back: 5.9 us; a
  // store, and a fence here, 6.0; the fence right behind the store 6.4.)
  auto settle = [&]() {
    if (was == 0x7fffffff) __nanosleep(0);
  };
  if (n <= p.budget) {  // (the whole cluster)
    settle();
    return;
  }
  const int last = max(p.q_pos ? p.q_pos[b] : n - 1, -1);
  const int recent = last - p.n_recent;  // positions above it are guarded
  const int per = (n + C - 1) / C;
  const int i0 = min(n, rank * per), cnt = min(n, i0 + per) - i0;  // this CTA's tokens
  const int32_t* table = p.g.block_table + (size_t)b * p.g.max_pages_per_seq;
  const bool held = per <= p.smem_keys;
  const int shrink = n - p.budget;

  auto slot_of = [&](int t) -> int {  // slot of the [page][head][row] pools; -1: not a page
    const int page = table[t >> shift];
    if (!page_ok(p.g, page)) return -1;
    return (page * H + head) * ps + (t & (ps - 1));
  };
  auto key_of = [&](int at, int pos, float w) -> uint32_t {
    if (at < 0) return 0u;
    return (pos < p.n_sink || pos > recent) ? 0xffffffffu : weight_key(w);
  };
  auto load_key = [&](int i) -> uint32_t {
    const int at = slot_of(i0 + i);
    return at < 0 ? 0u : key_of(at, p.positions[at], p.weights[at]);
  };
  auto key_at = [&](int i) -> uint32_t { return held ? keys[i] : load_key(i); };
  // visits every key of the CTA's share once, four loads in flight
  auto for_keys = [&](auto&& visit) {
    int bad = 0;
    for (int i = tid; i < cnt; i += 4 * kEvThreads) {
      int at[4], pos[4];
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) at[k] = i + k * kEvThreads < cnt ? slot_of(i0 + i + k * kEvThreads) : -2;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        pos[k] = at[k] >= 0 ? p.positions[at[k]] : 0;
        w[k] = at[k] >= 0 ? p.weights[at[k]] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bad |= at[k] == -1 ? 1 : 0;
        if (at[k] > -2) visit(i + k * kEvThreads, key_of(at[k], pos[k], w[k]));
      }
    }
    if (bad) atomicOr(p.status, MC_FLAG_BAD_METADATA);
  };
  auto copy_row = [&](int from, int to) {  // by a warp: lanes 0..15 K, 16..31 V
    char* pool = lane < 16 ? p.k_pool : p.v_pool;
    const uint4 v = ld_stream16(pool + (size_t)from * kRowBytes + (lane & 15) * 16);
    st_stream16(pool + (size_t)to * kRowBytes + (lane & 15) * 16, v);
  };

  if (shrink == 1 && C == 1) {
    // ---- one token too many: the smallest key, the last index among equals, goes; the last token takes its slot
    uint64_t best = ~0ull;  // (key, n - index): ties go to the lower index, so the higher one is evicted
    for_keys([&](int i, uint32_t k) { best = min(best, ((uint64_t)k << 32) | (uint32_t)(n - 1 - i)); });
#pragma unroll
    for (int o = 16; o; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) best_s[warp] = best;
    __syncthreads();
    if (warp != 0) {
      settle();
      return;
    }
    best = best_s[lane & (kEvWarps - 1)];
#pragma unroll
    for (int o = 16; o; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
    const int gone = n - 1 - (int)(uint32_t)best;
    if (gone == p.budget) return;  // the last token itself
    const int from = slot_of(p.budget), to = slot_of(gone);
    if (from < 0 || to < 0) return;
    copy_row(from, to);
    if (lane == 0) {
      p.weights[to] = p.weights[from];
      p.positions[to] = p.positions[from];
    }
    return;
  }

  for (int i = tid; i < kEvBins; i += kEvThreads) reinterpret_cast<uint4*>(total)[i] = make_uint4(0u, 0u, 0u, 0u);  // 3 totals, local
  if (C > 1) cl.sync();  // nobody adds to a total before it is cleared
  else __syncthreads();
  // ---- the budget-th largest key ------------------------------------------------------------------
  uint32_t prefix = 0;       // digits found so far
  int want = p.budget;       // rank of the key among those that share the prefix
#pragma unroll
  for (int d = 0; d < 3; ++d) {
    const int sh = d == 0 ? 21 : (d == 1 ? 10 : 0), bits = d == 2 ? 10 : 11;
    uint32_t* tot = total + d * kEvBins;
    uint32_t* h = C > 1 ? local : tot;
    auto count = [&](int i, uint32_t k) {
      if (d == 0 && held) keys[i] = k;
      if (d == 0 || (k >> ((sh + bits) & 31)) == prefix) atomicAdd(&h[(k >> sh) & ((1u << bits) - 1)], 1u);
    };
    if (d == 0 || !held) for_keys(count);
    else
      for (int i = tid; i < cnt; i += kEvThreads) count(i, keys[i]);
    __syncthreads();
    // a thread takes four digits, the largest first
    const int quad = kEvThreads - 1 - tid;
    const uint4 mine = reinterpret_cast<const uint4*>(h)[quad];
    if (C > 1) {
      reinterpret_cast<uint4*>(h)[quad] = make_uint4(0u, 0u, 0u, 0u);
      const uint32_t v[4] = {mine.x, mine.y, mine.z, mine.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (v[k])
          for (int r = 0; r < C; ++r) atomicAdd(cl.map_shared_rank(tot, r) + 4 * quad + k, v[k]);
      cl.sync();
    }
    const uint4 all = C > 1 ? reinterpret_cast<const uint4*>(tot)[quad] : mine;
    const int c4[4] = {(int)all.w, (int)all.z, (int)all.y, (int)all.x};
    const int sum = c4[0] + c4[1] + c4[2] + c4[3];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    Two all_sum;
    const Two before = warp_prefix({__shfl_sync(0xffffffffu, incl, 31), 0}, warp_s, warp, lane, all_sum);
    int above = before.a + incl - sum;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (above < want && want <= above + c4[k]) {
        found[0] = 4 * quad + 3 - k;
        found[1] = above;
        found[2] = c4[k];
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
  int tie = -0x40000000;  // ties before this warp's run; (all of them stay: no need to count)
  if (want < found[2]) {
    int ties = 0;
    for (int w = w0; w < w1; ++w) {
      const int i = 32 * w + lane;
      ties += __popc(__ballot_sync(0xffffffffu, i < cnt && key_at(i) == thr));
    }
    Two sum;
    tie = warp_prefix({ties, 0}, warp_s, warp, lane, sum).a;
    if (C > 1) {
      if (tid < C) cl.map_shared_rank(pub_tie, tid)[rank].a = sum.a;
      cl.sync();
      for (int r = 0; r < rank; ++r) tie += pub_tie[r].a;
    }
  }
  // ---- who stays; holes before the budget, movers behind it ------------------------------------------
  const bool all_ties = want >= found[2];
  auto stay_word = [&](int w, int& t) -> uint32_t {
    const int i = 32 * w + lane;
    const uint32_t k = i < cnt ? key_at(i) : 0u;
    if (all_ties) return __ballot_sync(0xffffffffu, i < cnt && k >= thr);
    const uint32_t eq = __ballot_sync(0xffffffffu, i < cnt && k == thr);
    const bool stay = i < cnt && (k > thr || (k == thr && t + __popc(eq & ((1u << lane) - 1u)) < want));
    t += __popc(eq);
    return __ballot_sync(0xffffffffu, stay);
  };
  // 32 words of the run, a lane each: what follows from a word is worked out for 32 of them at once
  auto stay_words = [&](int wb, int& t) -> uint32_t {
    uint32_t own = 0;
    const int live = min(32, w1 - wb);
#pragma unroll 4
    for (int j = 0; j < live; ++j) {
      const uint32_t s = stay_word(wb + j, t);
      if (lane == j) own = s;
    }
    return own;
  };
  auto split_word = [&](int w, uint32_t s, uint32_t& holes, uint32_t& movers) {
    const int rel = p.budget - (i0 + 32 * w), valid = w < w1 ? cnt - 32 * w : 0;  // tokens of the word before the budget; in all
    const uint32_t low = rel >= 32 ? 0xffffffffu : (rel <= 0 ? 0u : (1u << rel) - 1u);
    const uint32_t here = valid >= 32 ? 0xffffffffu : (valid <= 0 ? 0u : (1u << valid) - 1u);
    holes = ~s & low & here;
    movers = s & ~low & here;
  };
  Two mine = {0, 0};  // holes, movers
  int tie_w = tie;
  for (int wb = w0; wb < w1; wb += 32) {
    const uint32_t s = stay_words(wb, tie_w);
    if (held && wb + lane < w1) mask[wb + lane] = s;
    uint32_t holes, movers;
    split_word(wb + lane, s, holes, movers);
    mine.a += __popc(holes);
    mine.b += __popc(movers);
  }
  mine.a = __reduce_add_sync(0xffffffffu, mine.a);
  mine.b = __reduce_add_sync(0xffffffffu, mine.b);
  Two sum;
  Two at = warp_prefix(mine, warp_s, warp, lane, sum);
  int n_moves = sum.b;
  if (C > 1) {
    if (tid < C) cl.map_shared_rank(pub, tid)[rank] = sum;
    cl.sync();
    n_moves = 0;
    for (int r = 0; r < C; ++r) {
      const Two q = pub[r];
      if (r < rank) {
        at.a += q.a;
        at.b += q.b;
      }
      n_moves += q.b;
    }
  }
  int32_t* hole_l = p.lists + (size_t)seg * 2 * p.list_stride;
  int32_t* move_l = hole_l + p.list_stride;
  for (int wb = w0; wb < w1; wb += 32) {
    const uint32_t s = !held ? stay_words(wb, tie) : (wb + lane < w1 ? mask[wb + lane] : 0u);
    uint32_t holes, movers;
    split_word(wb + lane, s, holes, movers);
    const int both = __popc(holes) | __popc(movers) << 16;  // (sums of 32 words: at most 1024 each)
    int incl = both;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const uint32_t lt = (1u << lane) - 1u;
    const int live = min(32, w1 - wb), t0 = i0 + 32 * wb + lane;
    for (int j = 0; j < live; ++j) {
      const uint32_t hb = __shfl_sync(0xffffffffu, holes, j), mb = __shfl_sync(0xffffffffu, movers, j);
      const int ahead = __shfl_sync(0xffffffffu, incl - both, j);
      if ((hb >> lane) & 1u) hole_l[at.a + (ahead & 0xffff) + __popc(hb & lt)] = t0 + 32 * j;
      if ((mb >> lane) & 1u) move_l[at.b + (ahead >> 16) + __popc(mb & lt)] = t0 + 32 * j;
    }
    const int sums = __shfl_sync(0xffffffffu, incl, 31);
    at.a += sums & 0xffff;
    at.b += sums >> 16;
  }
  if (C > 1) cl.sync();  // the lists are complete (and nobody touches another CTA's shared memory from here on)
  else __syncthreads();
  // ---- the rows: a lane works a move's slots out, then the warp copies it ------------------------------
  const int n_warps = C * kEvWarps, gw = rank * kEvWarps + warp;
  const int rounds = (n_moves + 32 * n_warps - 1) / (32 * n_warps);  // equal shares, at most 32 moves at a time
  const int share = max(1, (n_moves + n_warps * rounds - 1) / max(n_warps * rounds, 1));
  char* pool = lane < 16 ? p.k_pool : p.v_pool;
  constexpr int kDeep = 4;  // rows in flight per warp (8: 8 % slower, 12: 22 %: too many open rows of memory)
  for (int m0 = gw * share; m0 < n_moves; m0 += n_warps * share) {
    const int m = m0 + lane;
    int src = -1, dst = -1;
    if (lane < share && m < n_moves) {
      src = slot_of(__ldcg(move_l + m));
      dst = slot_of(__ldcg(hole_l + m));
      if (src >= 0 && dst >= 0) {
        p.weights[dst] = p.weights[src];
        p.positions[dst] = p.positions[src];
      }
    }
    const int live = min(share, n_moves - m0);
    for (int k0 = 0; k0 < live; k0 += kDeep) {
      uint4 v[kDeep];
      int to[kDeep];
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int from = __shfl_sync(0xffffffffu, src, (k0 + k) & 31);
        to[k] = __shfl_sync(0xffffffffu, dst, (k0 + k) & 31);
        if (k0 + k >= live || from < 0) to[k] = -1;
        if (to[k] >= 0) v[k] = ld_stream16(pool + (size_t)from * kRowBytes + (lane & 15) * 16);
      }
#pragma unroll
      for (int k = 0; k < kDeep; ++k)
        if (to[k] >= 0) st_stream16(pool + (size_t)to[k] * kRowBytes + (lane & 15) * 16, v[k]);
    }
  }
  settle();
}

// ---- host side ------------------------------------------------------------------------------------
static int evict_list_stride(const mc_batch* bt) { return (bt->max_seq_len + 1) / 2 + 1; }  // min(budget, n - budget) at most
size_t layer_evict_workspace_bytes(const mc_config* cfg, const mc_batch* bt) {
  return align_up((size_t)bt->batch * cfg->n_kv_heads * 2 * evict_list_stride(bt) * 4, 256);
}

static constexpr size_t evict_smem(int keys) { return (size_t)(4 * kEvBins + keys + keys / 32 + 1) * 4; }

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
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  // CTAs per segment: as many as the GPU takes at once (two per SM), if a CTA still has 1024 tokens.  (More of them run
  // in two waves: 256 segments of 4096 tokens took 90 us with two CTAs each, 67 with one.)
  int cluster = 1;
  while (cluster < kEvMaxCluster && (long long)bt->batch * cfg->n_kv_heads * cluster * 2 <= 2 * n_sm &&
         bt->max_seq_len > 1024 * cluster)
    cluster *= 2;
  const int per = (bt->max_seq_len + cluster - 1) / cluster;
  ep.smem_keys = std::min((per + 31) / 32 * 32, kEvSmemKeys);
  const size_t smem = evict_smem(ep.smem_keys);
  MC_CUDA_CHECK(allow_smem(layer_evict_kernel, evict_smem(kEvSmemKeys)));
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
