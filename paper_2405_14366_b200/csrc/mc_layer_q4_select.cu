// Which pages of a 4-bit layer are worth attending: per (sequence, kv head) those with the largest bound
//
//   sum_h sum_c max(q_hc lo_c, q_hc hi_c) = Q.zero + 15 P.scale,   Q = sum_h q_h,  P = sum_h max(q_h, 0)
//
// over the kv head's query heads h (lo = zero, hi = zero + 15 scale, scale > 0: what channel c of a key of the page can hold).
// The keys' group parameters are the bounds already: 512 of a page's 5120 bytes are read, nothing else of the cache.
// Sums are held in 64 bits: the last page in and the first one out differ by less than binary32 resolves often enough
// that the choice would hang on the order of a sum.  (256 products a page are 4 cycles of the SM's 64-bit units; the page's bytes
// take 22 at the memory's rate.  Conversions, at 16 an SM and cycle, took as long as all the rest: the operands are put
// together from their bits, see tiny_zero.)
// A cluster of CTAs per (sequence, kv head) forms the sums; their binary32 roundings, which keep the order, go to the first
// CTA's shared memory, where a radix select finds the last one in (512 pages and fewer: a count).  Pages that round alike
// there are told apart by the 64-bit sums, and equal ones by their index.
// Measured, from a CUDA graph: 19.2 us for 4 x 131060 tokens of 8 kv heads (67 MB: 10.3 us at a copy's rate; the sums and the launch
// take 15.3, then one CTA of a cluster's four selects), 8.0 us for 16 x 8192, 5.6 us for one sequence of 8200 tokens and 32 heads.
#include <algorithm>

#include "mc_kernels.h"
#include "mc_layer.h"
#include "mc_layer_q4.cuh"
#include "mc_layer_q4.h"

namespace mc {

constexpr int kLsThreads = 512;
constexpr int kLsWarps = kLsThreads / 32;
constexpr int kLsMaxCluster = 8;
constexpr int kLsBatch = 4;   // pages of a warp at a time
// batches of a warp in shared memory: one worked on, one on its way (16 warps then have 32 KB on their way; with three or four:
// 9.8, 10.3 us for 9.4 at 16 x 8192 tokens, 20.8, 21.3 for 20.2 at 4 x 131060)
constexpr int kLsStages = 2;
constexpr int kLsRing = kLsWarps * kLsStages * kLsBatch * kLqMetaBytes;
constexpr int kLsBins = 2048;

struct Q4SelectParams {
  Geom g;
  ScoreRule rule;
  const unsigned char* k_meta;
  int32_t* status;
  const char* q;
  int32_t* pages;
  int32_t* counts;
  unsigned long long* keys;  // [segment][key_stride]: the sums in an order that compares as integers
  int key_stride;
  int budget, n_sink, n_recent;
  int nq, n_q_heads;
  int cluster;
};

__device__ __forceinline__ uint32_t order32(float x) {
  const uint32_t b = __float_as_uint(x);
  return x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long order64(double x) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(x);
  return x != x ? 0ull : (b >> 63) ? ~b : b | (1ull << 63);
}
// 2^-1008 times the binary16 number in the high (low, positive) half of w, finite, as a double: its exponent and mantissa in
// their places, its exponent not rebased -- a subnormal number too, as both formats count those in the unit of their lowest
// binade.
__device__ __forceinline__ double tiny_zero(uint32_t w) { return __hiloint2double((int)((w & 0x80000000u) | ((w >> 6) & 0x01fffc00u)), 0); }
__device__ __forceinline__ double tiny_scale(uint32_t w) { return __hiloint2double((int)((w << 10) & 0x01fffc00u), 0); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_first_cta(uint32_t* smem, uint32_t v) {
  uint32_t a;  // (its address in the first CTA)
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(smem)));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

// The sum of the warps' numbers that `mine` asks for (of warp `lane`).
__device__ __forceinline__ int sum_of(const int* warps, bool mine) {
  const int lane = threadIdx.x & 31;
  return __reduce_add_sync(0xffffffffu, mine && lane < kLsWarps ? warps[lane] : 0);
}

template <int DT>
__global__ void __launch_bounds__(kLsThreads, 1) layer_q4_select_kernel(const __grid_constant__ Q4SelectParams p) {
  grid_dep_launch();
  extern __shared__ __align__(16) unsigned char select_smem[];
  uint32_t* keys_s = reinterpret_cast<uint32_t*>(select_smem + kLsRing);  // [pages] of the first CTA
  __shared__ uint32_t hist[kLsBins];
  __shared__ int scan_s[kLsWarps], ins_s[kLsWarps], ties_s[kLsWarps];
  __shared__ uint32_t pick_s[2][3];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads;
  const int rank = blockIdx.x % p.cluster, seg = blockIdx.x / p.cluster;
  const int b = seg / H, head = seg - b * H;
  cluster_arrive();  // (every CTA of the cluster runs before one writes to another)
  grid_dep_wait();   // queries, parameters: what the kernels ahead have written
  const int raw = __ldcg(p.g.seq_lens + b);
  if ((raw < 0 || raw > p.g.max_seq_len) && tid == 0) atomicOr(p.status, MC_FLAG_BAD_METADATA);
  const int n = min(max(raw, 0), p.g.max_seq_len), full = n / kLqPage;
  const PageView v = page_view(p.rule, b, n, n + 1, n);
  const int u = v.u, take = min(p.budget, u);
  if (head == 0 && rank == 0 && tid == 0) p.counts[b] = take;
  int32_t* list = p.pages + (size_t)seg * p.budget;
  cluster_wait();
  if (u <= p.budget) {  // (the whole cluster)
    if (rank == 0)
      for (int k = tid; k < u; k += kLsThreads) list[k] = v.page_of(k);
    return;
  }
  unsigned long long* keys = p.keys + (size_t)seg * p.key_stride;
  for (int i = tid; i < kLsBins; i += kLsThreads) hist[i] = 0;
  {
    double Q[4] = {}, P[4] = {};
    for (int h = 0; h < p.nq; ++h) {
      const uint2 w = *reinterpret_cast<const uint2*>(p.q + ((size_t)b * p.n_q_heads + head * p.nq + h) * kRowBytes + 8 * lane);
      const float2 x = Elem<DT>::unpack(w.x), y = Elem<DT>::unpack(w.y);
      const float f[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        Q[c] += (double)f[c];
        P[c] += f[c] < 0.f ? 0.0 : (double)f[c];  // (a NaN stays one)
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      P[c] *= 15.0 * 0x1p504;  // (what the tiny numbers lack is put back in two steps: 2^1008 times a query overflows)
      Q[c] *= 0x1p504;
    }
    // The warp's pages: batches of four, every (cluster * warps)-th.  A lane knows the page of one of the next 32 (eight batches), and
    // keeps the sum of one: what is done to a sum is done to 32 at a time (to each batch's four at once: 22.5 us for 20.2);
    // the next batch's parameters are on their way while one is worked on, each lane's 16 bytes of a page to where it reads them.
    const int step = p.cluster * kLsWarps * kLsBatch, first = (rank * kLsWarps + warp) * kLsBatch;
    auto pages_from = [&](int k) {  // lane: page lane % batch of the batch k + lane / batch * step
      const int at = k + lane / kLsBatch * step + lane % kLsBatch;
      if (at >= u) return 0;
      const int page = checked_page(p.g, b, v.page_of(at), p.status);
      return page < 0 ? 0 : page;
    };
    constexpr int kTurns = 32 / kLsBatch;
    int ids = pages_from(first), ids_next = pages_from(first + kTurns * step), turn = 0, k_ahead = first, slot = 0;
    const unsigned char* meta = p.k_meta + (size_t)head * kLqMetaBytes + 16 * lane;
    unsigned char* ring = select_smem + warp * (kLsStages * kLsBatch * kLqMetaBytes) + 16 * lane;
    const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
    int slot_ahead = 0, done = 0;
    double mine = 0.0;
    auto issue = [&]() {
      if (k_ahead < u) {
#pragma unroll
        for (int j = 0; j < kLsBatch; ++j) {
          const int page = __shfl_sync(0xffffffffu, ids, kLsBatch * turn + j);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring_s + (slot_ahead * kLsBatch + j) * kLqMetaBytes),
                       "l"(meta + (size_t)page * H * kLqMetaBytes)
                       : "memory");
        }
        if (++turn == kTurns) {
          turn = 0;
          ids = ids_next;
          ids_next = pages_from(k_ahead + (kTurns + 1) * step);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      k_ahead += step;
      slot_ahead = (slot_ahead + 1) % kLsStages;
    };
#pragma unroll
    for (int i = 0; i < kLsStages - 1; ++i) issue();
    for (int k0 = first; k0 < u; k0 += step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kLsStages - 2) : "memory");
      uint4 cur[kLsBatch];
#pragma unroll
      for (int j = 0; j < kLsBatch; ++j) cur[j] = *reinterpret_cast<const uint4*>(ring + (slot * kLsBatch + j) * kLqMetaBytes);
      slot = (slot + 1) % kLsStages;
      issue();  // (into the batch read before this one)
      double a[kLsBatch];
#pragma unroll
      for (int j = 0; j < kLsBatch; ++j) {
        const uint32_t w[4] = {cur[j].x, cur[j].y, cur[j].z, cur[j].w};
        double t = 0.0;
#pragma unroll
        for (int c = 0; c < 4; ++c) t = fma(P[c], tiny_scale(w[c]), fma(Q[c], tiny_zero(w[c]), t));
        a[j] = t;
      }
      // four sums over the warp, halving the pages a lane keeps: lane 8 j ends with page j
#pragma unroll
      for (int o = 16, c = kLsBatch / 2; c > 0; o >>= 1, c >>= 1) {
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int j = 0; j < c; ++j) {
          const double give = up ? a[j] : a[j + c], keep = up ? a[j + c] : a[j];
          a[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
#pragma unroll
      for (int o = kTurns / 2; o > 0; o >>= 1) a[0] += __shfl_xor_sync(0xffffffffu, a[0], o);
      // (the lanes from kTurns j on have page j)
      if (lane % kTurns == done) mine = a[0];
      if (++done == kTurns || k0 + step >= u) {
        const int k = k0 + (lane % kTurns - (done - 1)) * step + lane / kTurns;
        if (lane % kTurns < done && k < u) {
          const int page = v.page_of(k);
          const double x = mine * 0x1p504 + 0.0;  // (-0 counts as 0)
          const bool guarded = page < p.n_sink || page >= full - p.n_recent;
          keys[k] = guarded ? ~0ull : order64(x);
          store_first_cta(keys_s + k, guarded ? 0xffffffffu : order32((float)x));
        }
        done = 0;
      }
    }
  }
  cluster_arrive();
  cluster_wait();
  if (rank != 0) return;

  // ---- few pages, a thread each: its rank is the number of larger keys (512 comparisons are less than a pass over the digits);
  // those that are alike are told apart only where they are too many
  if (u <= kLsThreads) {
    bool in = false;
    uint32_t c = 0;
    int above = 0;
    const int u4 = u / 4 * 4;
    if (tid < u) {
      c = keys_s[tid];
#pragma unroll 16
      for (int k = 0; k < u4; k += 4) {
        const uint4 o = *reinterpret_cast<const uint4*>(keys_s + k);
        above += (o.x > c ? 1 : 0) + (o.y > c ? 1 : 0) + (o.z > c ? 1 : 0) + (o.w > c ? 1 : 0);
      }
      for (int k = u4; k < u; ++k) above += keys_s[k] > c ? 1 : 0;
      in = above < take;
    }
    if (__syncthreads_count(in) > take) {  // some of those that are alike in 32 bits
      if (in) {
        const unsigned long long d = keys[tid];
        for (int k = 0; k < u; ++k)
          if (keys_s[k] == c && k != tid) above += keys[k] > d || (keys[k] == d && k < tid) ? 1 : 0;
      }
      in = in && above < take;
    }
    const uint32_t bi = __ballot_sync(0xffffffffu, in);
    if (lane == 0) ins_s[warp] = __popc(bi);
    __syncthreads();
    const int before = __popc(bi & ((1u << lane) - 1u)) + sum_of(ins_s, lane < warp);
    if (in) list[before] = v.page_of(tid);
    return;
  }
  // ---- the last one in: digits of the 32-bit keys, then (of those that are alike in them) of the 64-bit ones
  uint32_t p32 = 0, m32 = 0;
  unsigned long long p64 = 0, m64 = 0;
  int need = take;   // of those that match the digits so far
  bool all = false;  // every one of them
  for (int pass = 0; pass < 9 && !all; ++pass) {
    const bool wide = pass >= 3;
    const int width = pass == 2 ? 10 : pass == 8 ? 9 : 11;
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : pass == 2 ? 0 : pass == 8 ? 0 : 53 - 11 * (pass - 3);
    for (int k = 4 * tid; k < u; k += 4 * kLsThreads) {
      const uint4 c4 = *reinterpret_cast<const uint4*>(keys_s + k);
      const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k + j >= u || (c[j] & m32) != p32) continue;
        if (wide && m64 != 0 && (keys[k + j] & m64) != p64) continue;
        atomicAdd(&hist[(wide ? (uint32_t)(keys[k + j] >> shift) : c[j] >> shift) & ((1u << width) - 1u)], 1u);
      }
    }
    __syncthreads();
    // the bin from the top in which the need-th lies: thread t has four of them
    constexpr int kOwn = kLsBins / kLsThreads;
    uint32_t own[kOwn], sum = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      own[j] = hist[tid * kOwn + j];
      hist[tid * kOwn + j] = 0;  // (for the next digit)
      sum += own[j];
    }
    uint32_t above = sum;  // bins of this thread and those behind it in the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t t = __shfl_down_sync(0xffffffffu, above, o);
      if (lane + o < 32) above += t;
    }
    if (lane == 0) scan_s[warp] = (int)above;
    __syncthreads();
    above += sum_of(scan_s, lane > warp) - sum;
    if (above < (uint32_t)need && above + sum >= (uint32_t)need) {
#pragma unroll
      for (int j = kOwn - 1; j >= 0; --j) {
        if (above < (uint32_t)need && above + own[j] >= (uint32_t)need) {
          pick_s[pass & 1][0] = tid * kOwn + j;
          pick_s[pass & 1][1] = need - above;
          pick_s[pass & 1][2] = own[j];
        }
        above += own[j];
      }
    }
    __syncthreads();
    const uint32_t* pick = pick_s[pass & 1];
    const unsigned long long digit = pick[0], mask = (1u << width) - 1u;
    if (wide) {
      p64 |= digit << shift;
      m64 |= mask << shift;
    } else {
      p32 |= (uint32_t)digit << shift;
      m32 |= (uint32_t)mask << shift;
    }
    need = pick[1];
    all = pick[1] == pick[2];
  }

  // ---- the list, in ascending order: a warp has a run of pages, a lane at last 32 of it
  static_assert(kQ4MaxSelectLen / kLqPage <= kLsThreads * 32, "a lane has a word of them");
  const int per = ((u + kLsWarps - 1) / kLsWarps + 31) / 32 * 32;
  const int k0 = min(warp * per, u), k1 = min(k0 + per, u);
  uint32_t ins = 0, ties = 0;  // bit i: page k0 + 32 lane + i is above the border, or one of those on it
#pragma unroll 4
  for (int it = 0; it < per / 32; ++it) {
    const int k = k0 + 32 * it + lane;
    bool in = false, tie = false;
    if (k < k1) {
      const uint32_t c = keys_s[k] & m32;
      if (c != p32) {
        in = c > p32;
      } else if (m64 != 0) {
        const unsigned long long d = keys[k] & m64;
        in = d > p64;
        tie = d == p64;
      } else {
        tie = true;
      }
    }
    const uint32_t bi = __ballot_sync(0xffffffffu, in), bt = __ballot_sync(0xffffffffu, tie);
    if (lane == it) {
      ins = bi;
      ties = bt;
    }
  }
  const int n_in = __popc(ins), n_tie = __popc(ties);
  int in_before = n_in, tie_before = n_tie;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, in_before, o), y = __shfl_up_sync(0xffffffffu, tie_before, o);
    if (lane >= o) {
      in_before += x;
      tie_before += y;
    }
  }
  if (lane == 31) {
    ins_s[warp] = in_before;
    ties_s[warp] = tie_before;
  }
  __syncthreads();
  in_before += sum_of(ins_s, lane < warp) - n_in;
  tie_before += sum_of(ties_s, lane < warp) - n_tie;
  for (uint32_t left = ins | ties; left != 0; left &= left - 1) {
    const int i = __ffs(left) - 1;
    const bool in = (ins >> i) & 1u;
    if (in || tie_before < need)  // (the first `need` of the ties are in)
      list[in_before + min(tie_before, need)] = v.page_of(k0 + 32 * lane + i);
    in_before += in ? 1 : 0;
    tie_before += in ? 0 : 1;
  }
}

// ---- host side ------------------------------------------------------------------------------------
size_t layer_q4_select_workspace_bytes(const mc_config* cfg, const mc_batch* bt) {
  return align_up((size_t)bt->batch * cfg->n_kv_heads * (bt->max_seq_len / kLqPage) * 8, 256);
}

mc_status launch_layer_q4_select(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer,
                                 const mc_score_opts* opts, const mc_page_selection* keep, const void* q, int32_t* pages, int32_t* counts,
                                 void* workspace, cudaStream_t stream) {
  if (bt->batch == 0) return MC_OK;
  Q4SelectParams sp;
  sp.g = g;
  sp.rule = make_score_rule(opts);
  sp.k_meta = (const unsigned char*)layer->k_meta;
  sp.status = layer->status;
  sp.q = (const char*)q;
  sp.pages = pages;
  sp.counts = counts;
  sp.keys = (unsigned long long*)workspace;
  sp.key_stride = bt->max_seq_len / kLqPage;
  sp.budget = keep->budget;
  sp.n_sink = keep->n_sink;
  sp.n_recent = keep->n_recent;
  sp.nq = cfg->n_q_heads / cfg->n_kv_heads;
  sp.n_q_heads = cfg->n_q_heads;
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  // CTAs per (sequence, kv head): while all have an SM each and still a turn of pages for every warp
  const long long segs = (long long)bt->batch * cfg->n_kv_heads;
  int cluster = 1;
  while (cluster < kLsMaxCluster && segs * cluster * 2 <= n_sm && sp.key_stride >= 2 * cluster * kLsWarps * kLsBatch) cluster *= 2;
  sp.cluster = cluster;
  auto* kernel = cfg->dtype == MC_F16 ? layer_q4_select_kernel<MC_F16> : layer_q4_select_kernel<MC_BF16>;
  MC_CUDA_CHECK(allow_smem(kernel, kLsRing + (size_t)kQ4MaxSelectLen / kLqPage * 4));
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)(segs * cluster));
  lc.blockDim = dim3(kLsThreads);
  lc.dynamicSmemBytes = kLsRing + align_up((size_t)sp.key_stride * 4, 16);
  lc.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  lc.attrs = attr;
  lc.numAttrs = 2;
  MC_CUDA_CHECK(cudaLaunchKernelEx(&lc, kernel, sp));
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
