// The attention weight that the last J queries of a prompt give to every cached token of one uncompressed layer:
// w_i (+)= sum over the queries and the heads of a kv head's group of softmax(s)_i.  What mc_layer_evict ranks a
// prompt's tokens by before the first decode step.
//
// The R = J * nq query rows of a kv head meet its cached keys twice, on the 5th-generation tensor cores, 128 tokens
// at a time:
//   pass 1   D[query row][token] = Q K^T: a thread owns a query row and runs along the tokens, so the running maximum
//            and sum need no exchange between lanes (rows are laid out `rep` times over the 128 lanes when there are
//            few of them, each copy taking a share of the columns); partial (m, l) per (CTA, segment)
//   pass 2   D[token][query row] = K Q^T: the same two tiles with their roles exchanged; a thread owns a token and
//            sums 2^(s - lse) over the rows: no exchange either
// Keys are read twice and scores formed twice because a probability needs the whole row's sum first, and the scores of
// R rows (4 R bytes per token) are more to store and fetch than the key row (256 bytes).  Pass 2 walks its tiles
// backwards: the keys read last are the ones still in L2.
//
// Prompts that are short and few take another kernel, with the same two halves in one launch (layer_observe_short_kernel).
// One persistent CTA per SM; the tiles of all (sequence, kv head) segments are shared out equally.  The last warp streams
// K tiles (a tiled copy per page and 64-channel half), warp 0 the segments' Q; four groups of four warps take the scores
// out of tensor memory, each from a buffer of 128 columns of its own: up to 128 rows they take the tiles in turn, beyond
// that two of them share a tile, one per 128 rows.  Two threads issue tcgen05.mma, each for two groups: with one, a
// group that was late kept the others waiting for their next product.  Bounds: the keys' bytes, twice, and the 2 R
// exponentials per token (16 a clock and SM), with the cap's polynomial on the FMA pipe next to them.  Measured, from a CUDA
// graph: 168 us on 16 x 8192 tokens, 8 kv heads under 32, 32 queries, a cap (128 rows; 268 MB of keys: 3.2 TB/s over the two
// passes, 205 TFLOP/s); 195 us on 4 x 32749, 64 queries (256 rows; 352 TFLOP/s), of which the exponentials alone are 126.
// (Hundreds of passes back to back meet the power cap: 173 us at 1.84 GHz, 211 at 1.77, against 1.965.)
// Exactness: products and sums in binary32; exponentials to 2 ulp with results below 2^-126 flushed; the cap's tanh to 5e-8
// relative, its constants rounded once into the polynomial's coefficients.  Against 64 bits the weights are off by 1.7 times
// what elementary binary32 operations are.
// Every wait is bounded; tensor memory is taken behind the wait for the grid ahead and released on every path.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "mc_layer.cuh"
#include "mc_layer.h"
#include "mc_kernels.h"
#include "mc_pipe.cuh"
#include "mc_tc.cuh"

namespace mc {
namespace cg = cooperative_groups;

constexpr int kObTile = 128;                             // tokens per tile
constexpr int kObHalf = kObTile * 128;                   // bytes of a tile's 64-channel half
constexpr int kObTileBytes = 2 * kObHalf;                // 32 KB
constexpr int kObGroups = 4;                             // groups of four warps that take scores out of tensor memory
constexpr int kObChunk = 16;                             // columns in registers at a time
constexpr int kObThreads = 128 + kObGroups * 128;        // Q copies, tensor-core issue, the groups, tensor-core issue, K copies
constexpr int kObQBufs = 2;
constexpr int kObMaxStages = 4;
constexpr int kObNoToken = 0x7fffffff;                   // position of a tile's rows behind the sequence: never seen
constexpr int kObSmem = kObQBufs * kObTileBytes + kObMaxStages * kObTileBytes;  // 192 KB: Q buffers, then the K ring

struct ObserveParams {
  Geom g;
  ScoreRule rule;
  const int32_t* positions;
  float* weights;
  int32_t* status;
  float* part_ml;  // [(CTA + segment)][rows][slots][2]
  int n_obs, nq;
  int rows;      // n_obs * nq
  int nq_shift;  // nq = 1, 2, 4 or 8
  int nt;        // row tiles of 128: 1 or 2
  int slots;     // groups that share a row tile in pass 1: 4 / nt
  int rp, rep;   // rows of a copy (32, 64 or 128), copies in a row tile
  int jt;        // queries per Q copy
  int stage_shift;  // K ring: 4 or 2 stages
  int add;       // pass 2 adds to the weights (else it writes them)
  int zero;      // pass 1 clears the weights first
  int n_ctas;
  // Capped scores as d Q(d^2) straight from d = q.k: the polynomials of tanh with sm / cap and cap log2(e) folded into
  // their coefficients, and the |d| up to which each of them, and any of them, holds.
  float tiny[5], small[7];
  float tiny_max, small_max, poly_max;
};

// A sequence as the call sees it: tiles that hold a token some query sees (the first `ua`, then those from `ub0`).  Every
// CTA keeps them in shared memory: a demand load takes microseconds behind the stream of keys.
struct ObSeq {
  int n, last;
  int ua, ub0, u;
  int prefix, doc;
};
__device__ __forceinline__ View ob_view(const ObserveParams& p, const ObSeq& s, int q_pos) {
  return View{q_pos, s.prefix, p.rule.window > 0 ? max(s.doc, q_pos - p.rule.window + 1) : s.doc};
}
__device__ __forceinline__ ObSeq ob_seq(const ObserveParams& p, int b, int& bad) {
  ObSeq s;
  const int raw = __ldcg(p.g.seq_lens + b);  // (from L2: an eviction ahead in the stream may just have written it)
  const int at = p.rule.q_pos ? p.rule.q_pos[b] : 0;
  s.prefix = p.rule.prefix_len ? p.rule.prefix_len[b] : 0;
  s.doc = p.rule.doc_start ? p.rule.doc_start[b] : 0;
  bad |= raw < 0 || raw > p.g.max_seq_len ? 1 : 0;
  s.n = min(max(raw, 0), p.g.max_seq_len);
  s.last = min(max(p.rule.q_pos ? at : s.n - 1, -1), kObNoToken - 1);
  s.ua = (s.n + kObTile - 1) / kObTile;
  s.ub0 = s.u = s.ua;
  if (p.positions == nullptr) {
    const View first = ob_view(p, s, max(s.last - p.n_obs + 1, -1));  // the query that looks back furthest
    const int end = min(s.n - 1, s.last) + 1;
    const int a = max(min(end, first.prefix), 0), lo = max(first.lo_pos, a);
    s.ua = (a + kObTile - 1) / kObTile;
    s.ub0 = s.ua;
    int ub1 = s.ua;
    if (end > lo) {
      s.ub0 = max(lo / kObTile, s.ua);
      ub1 = max((end + kObTile - 1) / kObTile, s.ub0);
    }
    s.u = s.ua + ub1 - s.ub0;
  }
  return s;
}

// Where a role stands in its CTA's run of tiles.
struct ObCursor {
  int b, g, k, u;  // sequence, kv head, tile of the segment, tiles of the segment
  __device__ __forceinline__ void seek(const int* pre, int batch, int H, int x) {
    int lo = 0, hi = batch - 1;  // last b with pre[b] <= x
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pre[mid] <= x) lo = mid; else hi = mid - 1;
    }
    b = lo;
    u = (pre[b + 1] - pre[b]) / H;
    const int rem = x - pre[b];
    g = rem / u;
    k = rem - g * u;
  }
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void group_sync(int grp) { asm volatile("bar.sync %0, 128;" ::"r"(1 + grp) : "memory"); }
__device__ __forceinline__ void pair_sync(int pair) { asm volatile("bar.sync %0, 256;" ::"r"(1 + kObGroups + pair) : "memory"); }

__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[16]) {
  tmem_ld16_async(addr, r);
  tmem_wait16(r);
}
// c[0] + c[1] z + ... of two numbers.
template <int N>
__device__ __forceinline__ uint64_t poly(const float (&c)[N], uint64_t z) {
  uint64_t q = pack2(c[N - 1], c[N - 1]);
#pragma unroll
  for (int j = N - 2; j >= 0; --j) q = fma2(q, z, pack2(c[j], c[j]));
  return q;
}
__device__ __forceinline__ uint64_t choose(bool first_a, bool first_b, uint64_t x, uint64_t y) {
  float xa, xb, ya, yb;
  unpack2(x, xa, xb);
  unpack2(y, ya, yb);
  return pack2(first_a ? xa : ya, first_b ? xb : yb);
}
// Accumulators d -> factors t with score = d t (log2 units), two per 64-bit register: the scale, or the folded polynomial
// of the cap (d may be replaced: beyond the polynomials' range the score itself goes there, with factor 1).
template <bool CAP>
__device__ __forceinline__ void factors(const ObserveParams& p, uint32_t (&raw)[kObChunk], uint64_t (&t)[kObChunk / 2]) {
  if (!CAP) {
#pragma unroll
    for (int k = 0; k < kObChunk / 2; ++k) t[k] = pack2(p.rule.scale_log2, p.rule.scale_log2);
    return;
  }
  float big = 0.f;
#pragma unroll
  for (int k = 0; k < kObChunk; k += 2) big = max3_abs(big, __uint_as_float(raw[k]), __uint_as_float(raw[k + 1]));
  // Which form an accumulator takes follows from its own magnitude, as the forms differ in their last bits and most warps
  // hold accumulators that do not count (hidden, stale); the vote only spares the warp the forms that none of its
  // accumulators takes.  (A NaN is dropped by the maximum and stays one in every form.  One form for the whole warp, with
  // what does not count masked ahead of the vote, took 187 us on 16 x 8192 tokens, 8 kv heads under 32 and 32 queries, from
  // the registers that the masks need, and 157 with the vote alone; this takes 155, 168 instead of 164 where scores reach
  // half the cap, and up to 13 % more where most of them lie beyond it.)
  if (__all_sync(0xffffffffu, big <= p.tiny_max)) {
#pragma unroll
    for (int k = 0; k < kObChunk / 2; ++k) {
      const uint64_t d = pack2(__uint_as_float(raw[2 * k]), __uint_as_float(raw[2 * k + 1]));
      t[k] = poly(p.tiny, mul2(d, d));
    }
  } else if (__all_sync(0xffffffffu, big <= p.small_max)) {
#pragma unroll
    for (int k = 0; k < kObChunk / 2; ++k) {
      const float a = __uint_as_float(raw[2 * k]), b = __uint_as_float(raw[2 * k + 1]);
      const uint64_t d = pack2(a, b), z = mul2(d, d);
      t[k] = choose(fabsf(a) <= p.tiny_max, fabsf(b) <= p.tiny_max, poly(p.tiny, z), poly(p.small, z));
    }
  } else {
#pragma unroll
    for (int k = 0; k < kObChunk / 2; ++k) {
      const float a = __uint_as_float(raw[2 * k]), b = __uint_as_float(raw[2 * k + 1]);
      const uint64_t d = pack2(a, b), z = mul2(d, d);
      const bool near_a = fabsf(a) <= p.poly_max, near_b = fabsf(b) <= p.poly_max;
      const uint64_t q = choose(fabsf(a) <= p.tiny_max, fabsf(b) <= p.tiny_max, poly(p.tiny, z), poly(p.small, z));
      const float sa = score_of(p.rule, a), sb = score_of(p.rule, b);
      t[k] = choose(near_a, near_b, q, pack2(1.f, 1.f));
      raw[2 * k] = __float_as_uint(near_a ? a : sa);
      raw[2 * k + 1] = __float_as_uint(near_b ? b : sb);
    }
  }
}
// 2^x of two numbers.  (Taking three pairs in eight by a polynomial on the FMA pipe instead of the special-function unit
// lost 10 % on 256 uncapped rows: the warps wait for latencies, not for that unit.)
__device__ __forceinline__ uint64_t ex2_both(uint64_t x) {
  float a, b;
  unpack2(x, a, b);
  return pack2(ex2(a), ex2(b));
}

// Pass 1: 16 columns (tokens at `pos`, looked at unless the tile is seen whole) of this thread's query row.
template <bool CAP>
__device__ __forceinline__ void add_columns(const ObserveParams& p, uint32_t (&raw)[kObChunk], bool easy, const int* pos, const View& vw,
                                            float slope, bool no_max, float& m, uint64_t& lr) {
  uint64_t f[kObChunk / 2];
  factors<CAP>(p, raw, f);
  if (!easy) {  // distance bias and masks: the scores themselves, factor 1
#pragma unroll
    for (int k = 0; k < kObChunk; ++k) {
      const int pk = pos[k];
      float fa, fb;
      unpack2(f[k / 2], fa, fb);
      const float s = __uint_as_float(raw[k]) * ((k & 1) ? fb : fa);
      raw[k] = __float_as_uint(vw.sees(pk) ? fmaf(-slope, (float)(vw.q_pos - pk), s) : -INFINITY);
      if (k & 1) f[k / 2] = pack2(1.f, 1.f);
    }
  }
  if (!no_max) {
    float mx;
    if (CAP) {
      float s[kObChunk];
#pragma unroll
      for (int k = 0; k < kObChunk; k += 2)
        unpack2(mul2(pack2(__uint_as_float(raw[k]), __uint_as_float(raw[k + 1])), f[k / 2]), s[k], s[k + 1]);
      mx = s[0];
#pragma unroll
      for (int k = 1; k < kObChunk; ++k) mx = fmaxf(mx, s[k]);
    } else {
      const float scale = easy ? p.rule.scale_log2 : 1.f;
      mx = __uint_as_float(raw[0]);
      if (scale >= 0.f) {
#pragma unroll
        for (int k = 1; k < kObChunk - 1; k += 2) mx = max3(mx, __uint_as_float(raw[k]), __uint_as_float(raw[k + 1]));
        mx = fmaxf(mx, __uint_as_float(raw[kObChunk - 1]));
      } else {
#pragma unroll
        for (int k = 1; k < kObChunk; ++k) mx = fminf(mx, __uint_as_float(raw[k]));
      }
      mx *= scale;
    }
    if (mx > m) {
      const float g = ex2(m - mx);  // (l = 0 while m = -inf)
      lr = mul2(lr, pack2(g, g));
      m = mx;
    }
  }
  const float mb = m == -INFINITY ? 0.f : m;
  const uint64_t n2 = pack2(-mb, -mb);
  uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
  for (int k = 0; k < kObChunk; k += 4) {
    sum0 = add2(sum0, ex2_both(fma2(pack2(__uint_as_float(raw[k]), __uint_as_float(raw[k + 1])), f[k / 2], n2)));
    sum1 = add2(sum1, ex2_both(fma2(pack2(__uint_as_float(raw[k + 2]), __uint_as_float(raw[k + 3])), f[k / 2 + 1], n2)));
  }
  lr = add2(lr, add2(sum0, sum1));
}
// Pass 2: 16 query rows of this thread's token at `pos`, whose -log-sum-exps z2 holds.
struct ObRows {
  const float* neg_lse;
  const float* slope;
  const int* q_pos;
  const int* lo_pos;
  int live, prefix;
};
template <bool CAP>
__device__ __forceinline__ void add_rows(const ObserveParams& p, uint32_t (&raw)[kObChunk], const ulonglong2 (&z2)[kObChunk / 4], bool easy,
                                         const ObRows& rows, int pos, uint64_t& wa, uint64_t& wb, float& w) {
  uint64_t f[kObChunk / 2];
  factors<CAP>(p, raw, f);
  if (easy && rows.live == kObChunk) {
#pragma unroll
    for (int k = 0; k < kObChunk; k += 4) {
      const ulonglong2 z = z2[k / 4];
      wa = add2(wa, ex2_both(fma2(pack2(__uint_as_float(raw[k]), __uint_as_float(raw[k + 1])), f[k / 2], z.x)));
      wb = add2(wb, ex2_both(fma2(pack2(__uint_as_float(raw[k + 2]), __uint_as_float(raw[k + 3])), f[k / 2 + 1], z.y)));
    }
  } else {
#pragma unroll
    for (int k = 0; k < kObChunk; ++k) {
      if (k < rows.live) {
        float fa, fb;
        unpack2(f[k / 2], fa, fb);
        const View v = {rows.q_pos[k], rows.prefix, rows.lo_pos[k]};
        const float e = fmaf(-rows.slope[k], (float)(v.q_pos - pos), fmaf(__uint_as_float(raw[k]), (k & 1) ? fb : fa, rows.neg_lse[k]));
        if (v.sees(pos)) w += ex2(e);
      }
    }
  }
}

template <int DT, int PASS, bool CAP>
__global__ void __launch_bounds__(kObThreads, 1)
layer_observe_kernel(const __grid_constant__ ObserveParams p, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_q) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  // barriers: K full / empty per stage, Q full / empty per buffer, accumulator full / empty per group
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kObSmem);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kObMaxStages + 4 + 2 * kObGroups);
  volatile int* s_abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* row_s = reinterpret_cast<float*>(tmem_slot + 4);             // [groups][128][2]: pass 1 (m, l) of the lanes; pass 2 -lse, slope
  int* view_s = reinterpret_cast<int*>(row_s + kObGroups * kObTile * 2);  // [groups][2][128]: pass 2: position, lowest position seen
  int* pos_s = view_s + kObGroups * kObTile * 2;                      // pass 1: [groups][128] positions; pass 2: [2 turns][groups][128] partial weights
  int* pre_s = pos_s + 2 * kObGroups * kObTile;                           // [batch + 1]
  ObSeq* seq_s = reinterpret_cast<ObSeq*>(pre_s + p.g.batch + 1);     // [batch]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads, ps = p.g.page_size, shift = p.g.page_shift;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kObMaxStages, qfull0 = empty0 + 8 * kObMaxStages, qempty0 = qfull0 + 16;
  const uint32_t tfull0 = qempty0 + 16, tempty0 = tfull0 + 8 * kObGroups;
  const int q_bytes = p.nt * kObTileBytes, q_half = p.nt * kObHalf;
  const uint32_t sq0 = smem_u32(smem), sk0 = sq0 + kObQBufs * q_bytes;
  constexpr uint32_t tmem_cols = kObGroups * kObTile;

  if (tid == kObThreads - 1) {
    prefetch_map(&map_k);
    prefetch_map(&map_q);
  }
  int bad = 0;
  for (int b = tid; b < p.g.batch; b += kObThreads) {
    const ObSeq s = ob_seq(p, b, bad);
    seq_s[b] = s;
    pre_s[b + 1] = s.u * H;
  }
  if (tid == 0) {
    for (int s = 0; s < kObMaxStages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, p.nt);  // both issuing threads read a tile that has two row tiles
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(qfull0 + 8 * s, 1);
      mbar_init(qempty0 + 8 * s, 2);
    }
    for (int s = 0; s < kObGroups; ++s) {
      mbar_init(tfull0 + 8 * s, 1);
      mbar_init(tempty0 + 8 * s, 4);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (warp == 0) {  // exclusive prefix of the sequences' tiles (all kv heads)
    const int per = (p.g.batch + 31) / 32;
    const int b0 = min(lane * per, p.g.batch), b1 = min(b0 + per, p.g.batch);
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += pre_s[b + 1];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    int acc = incl - sum;
    for (int b = b0; b < b1; ++b) {
      acc += pre_s[b + 1];
      pre_s[b + 1] = acc;
    }
    if (lane == 0) pre_s[0] = 0;
  }
  __syncthreads();
  const long long U = pre_s[p.g.batch];
  const int T = (int)min((long long)p.n_ctas, max(U, 1LL));  // no live CTA's share is empty
  const int cta = blockIdx.x;
  int x_begin = 0, n_x = 0;
  if (cta < T) {
    const bool small = U * T <= 0xffffffffLL;  // (64-bit division is a hundred instructions)
    x_begin = small ? (int)((uint32_t)U * (uint32_t)cta / (uint32_t)T) : (int)(U * cta / T);
    n_x = (small ? (int)((uint32_t)U * (uint32_t)(cta + 1) / (uint32_t)T) : (int)(U * (cta + 1) / T)) - x_begin;
  }
  constexpr int DIR = PASS == 1 ? 1 : -1;
  const int s_mask = (1 << p.stage_shift) - 1;
  const int x_first = PASS == 1 ? x_begin : x_begin + n_x - 1;
  // Rows of the pools where the pages of the next tiles begin, a lane per page, one window of 32 pages ahead: a load
  // per tile would pace the stream by its latency.
  const int ppt = kObTile >> shift, lane_tile = lane >> (7 - shift), lane_page = lane & (ppt - 1);
  const int win_tiles = 32 >> (7 - shift);  // pages per tile: ppt; tiles per window
  auto load_window = [&](int k0, int& head, bool& has) {
    const int i = k0 + lane_tile;
    head = 0;
    has = false;
    if (i >= n_x) return 0;
    ObCursor d;
    d.seek(pre_s, p.g.batch, H, x_first + DIR * i);
    const ObSeq& q = seq_s[d.b];
    const int t = (d.k < q.ua ? d.k : q.ub0 + d.k - q.ua) * kObTile + (lane_page << shift);
    head = d.g;
    has = t < q.n;
    return has ? p.g.block_table[(size_t)d.b * p.g.max_pages_per_seq + (t >> shift)] : 0;
  };
  int head = 0, head_n = 0, page = 0, page_n = 0;
  bool has = false, has_n = false;
  if (warp == 3 + 4 * kObGroups) {  // (the block table is the caller's: read before the wait)
    page = load_window(0, head, has);
    page_n = load_window(win_tiles, head_n, has_n);
  }
  grid_dep_wait();
  // Tensor memory is taken behind the wait -- held in front of it, it could be what a CTA of the grid ahead is waiting
  // for -- and dependents may start once it is ours: one that took it first would wait for this grid.
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_d = *tmem_slot;
  grid_dep_launch();
  if (bad) atomicOr(p.status, MC_FLAG_BAD_METADATA);

  if (PASS == 1 && p.zero) {  // tokens that no query sees keep no weight: all are cleared, pass 2 adds
    for (int s = cta; s < p.g.batch * H; s += gridDim.x) {
      const int b = s / H, g = s - b * H;
      const int n = seq_s[b].n;
      for (int t = tid; t < n; t += kObThreads) {
        const int page = p.g.block_table[(size_t)b * p.g.max_pages_per_seq + (t >> shift)];
        if (page_ok(p.g, page)) p.weights[((size_t)page * H + g) * ps + (t & (ps - 1))] = 0.f;
      }
    }
  }

  // the step from tile to tile; `seg` tells that the next tile begins another segment
  auto advance = [&](ObCursor& c, int x) {
    c.k += DIR;
    if ((unsigned)c.k >= (unsigned)c.u) c.seek(pre_s, p.g.batch, H, x);
  };
  auto last_of_seg = [&](const ObCursor& c, int i) { return i + 1 == n_x || (DIR > 0 ? c.k + 1 == c.u : c.k == 0); };

  if (warp == 0) {
    // ===================== Q of the segments =====================
    ObCursor c;
    if (n_x > 0) c.seek(pre_s, p.g.batch, H, x_first);
    int seg = 0;
    for (int i = 0; i < n_x;) {
      const int qb = seg & 1;
      bool ok = true;
      if (seg >= 2) ok = __all_sync(0xffffffffu, mbar_wait_lean(qempty0 + 8 * qb, ((seg >> 1) - 1) & 1, s_abort, p.status));
      if (!ok) break;
      if (lane == 0) {
        const uint32_t bar = qfull0 + 8 * qb, dst = sq0 + qb * q_bytes;
        mbar_expect_tx(bar, (uint32_t)(2 * p.nt * p.rep * p.jt * p.nq * 128));
        for (int tt = 0; tt < p.nt; ++tt)
          for (int r = 0; r < p.rep; ++r)
            for (int h = 0; h < 2; ++h)
              tma_load_3d(dst + h * q_half + (tt * kObTile + r * p.rp) * 128, &map_q, 64 * h, c.g * p.nq, c.b * p.n_obs + tt * p.jt, bar);
      }
      __syncwarp();
      ++seg;
      i += DIR > 0 ? c.u - c.k : c.k + 1;  // the first tile of the next segment
      if (i < n_x) c.seek(pre_s, p.g.batch, H, x_first + DIR * i);
    }
  } else if (warp == 3 + 4 * kObGroups) {
    // ===================== K tiles =====================
    for (int i = 0; i < n_x; ++i) {
      const int in_win = i & (win_tiles - 1);
      if (in_win == 0 && i > 0) {
        page = page_n;
        head = head_n;
        has = has_n;
        page_n = load_window(i + win_tiles, head_n, has_n);
      }
      const int s = i & s_mask, lap = i >> p.stage_shift;
      bool ok = true;
      if (lap > 0) ok = __all_sync(0xffffffffu, mbar_wait_lean(empty0 + 8 * s, (lap - 1) & 1, s_abort, p.status));
      if (!ok) break;
      const uint32_t bar = full0 + 8 * s, dst = sk0 + s * kObTileBytes;
      const bool copies = has && lane_tile == in_win;
      const int n_copy = __popc(__ballot_sync(0xffffffffu, copies));
      if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n_copy * 2 * ps * 128));
      __syncwarp();
      if (copies) {
        int pg = page;
        if (!page_ok(p.g, pg)) {  // never an address: page 0 is read in its place and the call flagged
          atomicOr(p.status, MC_FLAG_BAD_METADATA);
          pg = 0;
        }
        const int y = (pg * H + head) * ps;
        const uint32_t to = dst + lane_page * ps * 128;
        tma_load_2d(to, &map_k, 0, y, bar);
        tma_load_2d(to + kObHalf, &map_k, 64, y, bar);
      }
      __syncwarp();
    }
  } else if (warp == 1 || warp == 2 + 4 * kObGroups) {
    // ===================== tensor-core issue: thread 0 for groups 0 and 2, thread 1 for groups 1 and 3 =====================
    const int issuer = warp == 1 ? 0 : 1;
    if (lane == 0) {
      ObCursor c;
      if (n_x > 0) c.seek(pre_s, p.g.batch, H, x_first);
      int seg = 0;
      bool first = true;
      // A descriptor's low word is an address in 16-byte units (and fixed bits), its high word never changes; k step 4
      // starts the second 64-channel half.
      const uint64_t d0 = smem_desc_k128(0);
      const uint32_t d_hi = (uint32_t)(d0 >> 32), d_lo = (uint32_t)d0, q_step = (uint32_t)(q_half >> 4);
      const int tt = p.nt == 1 ? 0 : issuer;  // this thread's row tile
      const int n_cols = PASS == 1 ? kObTile : (min(p.rows - tt * kObTile, kObTile) + 15) / 16 * 16;
      const uint32_t idesc = umma_idesc<DT, 8>() - (1u << 17) + ((uint32_t)(n_cols >> 3) << 17);
      for (int i = 0; i < n_x; ++i) {
        const int s = i & s_mask, qb = seg & 1;
        if (first && !mbar_wait_lean(qfull0 + 8 * qb, (seg >> 1) & 1, s_abort, p.status)) break;
        if (p.nt == 2 || (i & 1) == issuer) {
          if (!mbar_wait_lean(full0 + 8 * s, (i >> p.stage_shift) & 1, s_abort, p.status)) break;
          const int grp = p.nt == 1 ? i & 3 : 2 * (i & 1) + tt, turn = p.nt == 1 ? i >> 2 : i >> 1;
          if (turn >= 1 && !mbar_wait_lean(tempty0 + 8 * grp, (turn - 1) & 1, s_abort, p.status)) break;
          tc_fence_after();
          const uint32_t q_lo = d_lo + ((sq0 + qb * q_bytes) >> 4) + (uint32_t)(tt * (kObHalf >> 4));
          const uint32_t k_lo = d_lo + ((sk0 + s * kObTileBytes) >> 4), d = tmem_d + grp * kObTile;
#pragma unroll
          for (int k = 0; k < kHeadDim / 16; ++k) {
            const uint32_t ql = q_lo + (k >= 4 ? q_step : 0u) + (uint32_t)(2 * (k & 3));
            const uint32_t kl = k_lo + (uint32_t)((k >> 2) * (kObHalf >> 4) + 2 * (k & 3));
            const uint64_t dq = ((uint64_t)d_hi << 32) | ql, dk = ((uint64_t)d_hi << 32) | kl;
            if (PASS == 1) umma_f16(d, dq, dk, idesc, k > 0 ? 1u : 0u);
            else umma_f16(d, dk, dq, idesc, k > 0 ? 1u : 0u);
          }
          umma_commit(tfull0 + 8 * grp);
          umma_commit(empty0 + 8 * s);
        }
        first = last_of_seg(c, i);
        if (first) {
          umma_commit(qempty0 + 8 * qb);  // (arrives at once if this thread had no tile of the segment)
          ++seg;
        }
        if (i + 1 < n_x) advance(c, x_first + DIR * (i + 1));
      }
    }
  } else {
    // ===================== scores =====================
    // with one row tile the group takes every fourth tile, with two every second one, the rows of tile `tt`
    const int grp = (warp - 2) >> 2, quad = warp & 3, gl = quad * 32 + lane;  // gl: this thread's tensor-memory lane
    const int tt = p.nt == 1 ? 0 : grp & 1, stride = 4 / p.nt, mine = p.nt == 1 ? grp : grp >> 1;
    const int row0 = tt * kObTile, n_rows = min(p.rows - row0, kObTile);
    const uint32_t tbuf = tmem_d + grp * kObTile + ((uint32_t)(quad * 32) << 16);
    const uint32_t my_full = tfull0 + 8 * grp, my_empty = tempty0 + 8 * grp;
    float* row_g = row_s + grp * kObTile * 2;
    int* row_q = view_s + grp * kObTile * 2;
    int* pos_g = pos_s + grp * kObTile;
    const bool no_max = CAP && p.rule.cap_log2 <= 100.f && p.rule.slopes == nullptr;
    // pass 1: this lane's row, and the columns its copy takes
    const int c_n = p.rp, c_lo = gl & ~(p.rp - 1), r_own = gl & (p.rp - 1);  // (copies of rp rows, 128 / rp of them: rp columns each)
    const bool live = r_own < n_rows, warp_live = ((quad * 32) & (p.rp - 1)) < n_rows;
    View v0 = {}, vw = {};  // of the first query; pass 1: of this lane's row
    float m = 0.f, l = 0.f, slope = 0.f;
    int n = 0, skip = 0, ua = 0, easy_hi = 0, easy_pre = 0, easy_lo = 0;  // of the segment
    const int32_t* table = p.g.block_table;
    ObCursor c = {-1, 0, 0, 0};

    auto begin_segment = [&]() {
      const ObSeq& sq = seq_s[c.b];
      n = sq.n;
      ua = sq.ua;
      skip = sq.ub0 - sq.ua;
      table = p.g.block_table + (size_t)c.b * p.g.max_pages_per_seq;
      v0 = ob_view(p, sq, max(sq.last - p.n_obs + 1, -1));
      const View v1 = ob_view(p, sq, sq.last);
      // a tile that every query sees whole needs no masks: t0 <= easy_hi and (t0 <= easy_pre or t0 >= easy_lo)
      easy_hi = p.positions || p.rule.slopes ? -1 : min(n, v0.q_pos + 1) - kObTile;
      easy_pre = v0.prefix - kObTile;
      easy_lo = v1.lo_pos;
      if (PASS == 1) {
        m = no_max ? 0.f : -INFINITY;
        l = 0.f;
        const int r = row0 + (live ? r_own : 0);
        vw = ob_view(p, sq, max(sq.last - p.n_obs + 1 + (r >> p.nq_shift), -1));
        slope = p.rule.slopes ? p.rule.slopes[c.g * p.nq + (r & (p.nq - 1))] * kLog2e : 0.f;
      } else {
        // -log-sum-exp of every row, from the partial sums of the CTAs (and their groups) that share the segment
        const long long x0 = pre_s[c.b] + (long long)c.g * c.u;
        const long long y0 = (x0 + 1) * T - 1, y1 = (x0 + c.u) * T - 1;
        const int c0 = y1 < 0xffffffffLL ? (int)((uint32_t)y0 / (uint32_t)U) : (int)(y0 / U);
        const int c1 = y1 < 0xffffffffLL ? (int)((uint32_t)y1 / (uint32_t)U) : (int)(y1 / U);
        group_sync(grp);  // everybody has done with the segment before
        if (gl < n_rows) {
          const int r = row0 + gl;
          float mm = -INFINITY, ll = 0.f;
          for (int cc = c0; cc <= c1; cc += 4) {  // the parts of four CTAs in flight
            float4 q[4][2];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              q[e][0] = q[e][1] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (cc + e > c1) continue;
              const float4* s4 = reinterpret_cast<const float4*>(p.part_ml + ((size_t)(cc + e + c.b * H + c.g) * p.rows + r) * p.slots * 2);
              q[e][0] = s4[0];
              if (p.slots == 4) q[e][1] = s4[1];
            }
            float M = mm;  // (a part without a token has sum 0 and counts for nothing)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                if (q[e][k].y == 0.f) q[e][k].x = -INFINITY;
                if (q[e][k].w == 0.f) q[e][k].z = -INFINITY;
                M = fmaxf(M, fmaxf(q[e][k].x, q[e][k].z));
              }
            ll = ll == 0.f ? 0.f : ll * ex2(mm - M);
            mm = M;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                if (q[e][k].y != 0.f) ll = fmaf(q[e][k].y, ex2(q[e][k].x - M), ll);
                if (q[e][k].w != 0.f) ll = fmaf(q[e][k].w, ex2(q[e][k].z - M), ll);
              }
          }
          row_g[gl] = ll == 0.f ? -INFINITY : -(mm + log2f(ll));  // (a row that saw nothing gives nothing)
          row_g[kObTile + gl] = p.rule.slopes ? p.rule.slopes[c.g * p.nq + (r & (p.nq - 1))] * kLog2e : 0.f;
          const View v = ob_view(p, sq, max(sq.last - p.n_obs + 1 + (r >> p.nq_shift), -1));
          row_q[gl] = v.q_pos;
          row_q[kObTile + gl] = v.lo_pos;
        }
        group_sync(grp);
      }
    };
    // Pass 1: a segment of the CTA in which this group had no tile has an empty part of it.  (`filled`: the next segment
    // without a part.  Clearing the CTA's parts beforehand took 5000 cycles before the first copy of keys.)
    int filled = 0;
    auto fill_to = [&](int seg) {
      for (; filled < seg; ++filled)
        if (gl < n_rows)
          reinterpret_cast<float2*>(p.part_ml)[((size_t)(cta + filled) * p.rows + row0 + gl) * p.slots + mine] = make_float2(0.f, 0.f);
    };
    auto end_segment = [&]() {  // pass 1: the copies of a row meet; one partial result per (CTA, segment, group)
      fill_to(c.b * H + c.g);
      ++filled;
      group_sync(grp);
      row_g[2 * gl] = l == 0.f ? -INFINITY : m;
      row_g[2 * gl + 1] = live ? l : 0.f;
      group_sync(grp);
      if (gl < p.rp && gl < n_rows) {
        float mm = -INFINITY, ll = 0.f;
        for (int k = 0; k < p.rep; ++k) {
          const float mk = row_g[2 * (k * p.rp + gl)], lk = row_g[2 * (k * p.rp + gl) + 1];
          const float M = fmaxf(mm, mk);
          ll = (ll == 0.f ? 0.f : ll * ex2(mm - M)) + (lk == 0.f ? 0.f : lk * ex2(mk - M));
          mm = M;
        }
        reinterpret_cast<float2*>(p.part_ml)[((size_t)(cta + c.b * H + c.g) * p.rows + row0 + gl) * p.slots + mine] = make_float2(mm, ll);
      }
    };

    if (PASS == 1 && n_x > 0) {
      ObCursor a;
      a.seek(pre_s, p.g.batch, H, x_begin);
      filled = a.b * H + a.g;
    }
    uint32_t turn = 0;  // tiles this group has taken
    for (int i = mine; i < n_x; i += stride, ++turn) {  // (to the end also after a wait that ran out: the barriers stay matched)
      if (c.b >= 0) c.k += DIR * stride;
      if ((unsigned)c.k >= (unsigned)c.u) {
        if (PASS == 1 && c.b >= 0) end_segment();
        c.seek(pre_s, p.g.batch, H, x_first + DIR * i);
        begin_segment();
      }
      const int t0 = (c.k < ua ? c.k : c.k + skip) * kObTile;
      const bool easy = t0 <= easy_hi && (t0 <= easy_pre || t0 >= easy_lo);
      // this thread's token: its page is asked for now; what follows from it, its position and (pass 2) where its weight
      // goes, is looked at only when needed: the load takes microseconds behind the stream of keys
      const int t = t0 + gl;
      int pos = t < n ? t : kObNoToken;
      const int page = (PASS == 2 || !easy) && t < n ? table[t >> shift] : -1;
      const int at = (page * H + c.g) * ps + (t & (ps - 1));
      if (p.positions && page_ok(p.g, page)) pos = p.positions[at];
      if (PASS == 1 && !easy) {
        group_sync(grp);
        pos_g[gl] = pos;
        group_sync(grp);
      }
      const bool good = __all_sync(0xffffffffu, mbar_wait_lean(my_full, turn & 1, s_abort, p.status));
      tc_fence_after();
      float w = 0.f;
      bool released = false;
      auto release = [&]() {  // the buffer, as soon as its last columns are in registers
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(my_empty);
        released = true;
      };
      if (good && PASS == 1 && warp_live) {
        uint64_t lr = pack2(l, 0.f);
#pragma unroll 1
        for (int ch = c_lo; ch < c_lo + c_n; ch += kObChunk) {
          uint32_t raw[kObChunk];
          tmem_load(tbuf + ch, raw);
          if (ch + kObChunk == c_lo + c_n) release();
          add_columns<CAP>(p, raw, easy, pos_g + ch, vw, slope, no_max, m, lr);
        }
        float la, lb;
        unpack2(lr, la, lb);
        l = la + lb;
      } else if (good && PASS == 2) {
        uint64_t wa = 0, wb = 0;
#pragma unroll 1
        for (int r0 = 0; r0 < n_rows; r0 += kObChunk) {
          uint32_t raw[kObChunk];
          tmem_ld16_async(tbuf + r0, raw);
          ulonglong2 z2[kObChunk / 4];  // -log-sum-exps, on their way together with the scores
#pragma unroll
          for (int k = 0; k < kObChunk / 4; ++k) z2[k] = reinterpret_cast<const ulonglong2*>(row_g + r0)[k];
          tmem_wait16(raw);
          if (r0 + kObChunk >= n_rows) release();
          const ObRows rows = {row_g + r0, row_g + kObTile + r0, row_q + r0, row_q + kObTile + r0, min(n_rows - r0, kObChunk), v0.prefix};
          add_rows<CAP>(p, raw, z2, easy, rows, pos, wa, wb, w);
        }
        float a0, a1, b0, b1;
        unpack2(wa, a0, a1);
        unpack2(wb, b0, b1);
        w += (a0 + a1) + (b0 + b1);
      }
      if (!released) release();
      if (PASS == 2) {
        if (p.nt == 2) {  // a token's partial weights meet; the next turn's barrier lies between this read and the slot's reuse
          float* part = reinterpret_cast<float*>(pos_s) + ((turn & 1) * kObGroups + grp - tt) * kObTile + gl;
          if (tt == 1) *part = w;
          pair_sync(grp >> 1);
          if (tt == 0) w += *part;
        }
        if (tt == 0 && page_ok(p.g, page)) p.weights[at] = (p.add ? p.weights[at] : 0.f) + w;
      }
    }
    if (PASS == 1 && n_x > 0) {
      if (c.b >= 0) end_segment();
      ObCursor z;
      z.seek(pre_s, p.g.batch, H, x_begin + n_x - 1);
      fill_to(z.b * H + z.g + 1);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*s_abort) {  // let copies in flight land before the CTA's memory is released
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
  if (warp == 1) tmem_dealloc(tmem_d, tmem_cols);
}

// ---- short prompts: both passes in one launch -------------------------------------------------------
// A cluster per (sequence, kv head); a CTA has one, two or four tiles of 128 tokens and reads their keys once.  Tensor
// memory holds four products of 128 rows: with room for both, pass 2's are issued at once (they need nothing from pass 1),
// else as soon as pass 1 is through with its own.  The four groups share out (tile, row tile) units, and a unit's columns
// or rows where there are fewer units than groups; the row sums of the CTAs meet through distributed shared memory between
// the two halves of the arithmetic.  Tiles are not left out here: one that no query sees gets its weights, zeros, from the
// CTA that has it.
constexpr int kOsMaxCluster = 8;
constexpr int kOsThreads = kObGroups * 128;
constexpr int kOsRows = 2 * kObTile;
constexpr int kOsMaxTiles = 4;  // of a CTA; times row tiles: at most 4 as well
constexpr int kOsArrays = kOsMaxCluster * kOsRows * 8 + kOsRows * 16 + kObGroups * kObTile * 8 + kOsMaxTiles * kObTile * 4 + kObGroups * kObTile * 4;

template <int DT, bool CAP, int T>
__global__ void __launch_bounds__(kOsThreads, 1)
layer_observe_short_kernel(const __grid_constant__ ObserveParams p, const __grid_constant__ CUtensorMap map_k,
                           const __grid_constant__ CUtensorMap map_q) {
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float2* all_s = reinterpret_cast<float2*>(smem + (T + p.nt) * kObTileBytes);  // [CTA of the cluster][rows] (m, l), written by the cluster
  float* neg_lse = reinterpret_cast<float*>(all_s + kOsMaxCluster * kOsRows);   // [rows], then slopes, positions, lowest positions seen
  float* slope_s = neg_lse + kOsRows;
  int* qpos_s = reinterpret_cast<int*>(slope_s + kOsRows);
  int* lo_s = qpos_s + kOsRows;
  float2* part_s = reinterpret_cast<float2*>(lo_s + kOsRows);  // [groups][128] (m, l) of the lanes
  int* pos_s = reinterpret_cast<int*>(part_s + kObGroups * kObTile);  // [tiles][128]
  float* w_s = reinterpret_cast<float*>(pos_s + T * kObTile);         // [groups][128]
  __shared__ uint64_t bars[3];  // operands, products of pass 1, of pass 2
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_s;
  volatile int* s_abort = &abort_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads, ps = p.g.page_size, shift = p.g.page_shift;
  const int seg = blockIdx.x / C, b = seg / H, head = seg - b * H;
  const uint32_t full = smem_u32(bars), done1 = full + 8, done2 = full + 16;
  const uint32_t sk = smem_u32(smem), sq = sk + T * kObTileBytes;
  const int q_half = p.nt * kObHalf;
  const int two = p.nt - 1, units = T << two;  // (1, 2 or 4)
  const bool both = T == 1 || units <= 2;
  const uint32_t tmem_cols = units == 1 ? 2 * kObTile : 4 * kObTile;

  if (tid == 0) {
    prefetch_map(&map_k);
    prefetch_map(&map_q);
    for (int k = 0; k < 3; ++k) mbar_init(full + 8 * k, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  int bad = 0;
  const ObSeq s = ob_seq(p, b, bad);
  const int t0 = rank * T * kObTile, n = s.n;
  const int live = min(T, max(n - t0 + kObTile - 1, 0) / kObTile);  // tiles with a token
  const int32_t* table = p.g.block_table + (size_t)b * p.g.max_pages_per_seq;
  // warp 0: the tiles' pages, a lane each (32 at most); a thread per token: its token's
  const bool has = warp == 0 && lane < T * (kObTile >> shift) && t0 + (lane << shift) < n;
  const int copy_page = has ? table[(t0 >> shift) + lane] : 0;
  const int page = tid < T * kObTile && t0 + tid < n ? table[(t0 + tid) >> shift] : -1;
  grid_dep_wait();
  // Tensor memory is taken behind the wait -- held in front of it, it could be what a CTA of the grid ahead is waiting
  // for -- while warp 0 issues the copies.
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), tmem_cols);
  if (live && warp == 0) {
    const int n_copy = __popc(__ballot_sync(0xffffffffu, has));
    if (lane == 0) mbar_expect_tx(full, (uint32_t)(n_copy * 2 * ps * 128 + 2 * p.nt * p.rep * p.jt * p.nq * 128));
    __syncwarp();
    if (has) {
      int pg = copy_page;
      if (!page_ok(p.g, pg)) {  // never an address: page 0 is read in its place and the call flagged
        atomicOr(p.status, MC_FLAG_BAD_METADATA);
        pg = 0;
      }
      const int y = (pg * H + head) * ps;
      const int j = (lane << shift) / kObTile;
      const uint32_t to = sk + j * kObTileBytes + ((lane << shift) - j * kObTile) * 128;
      tma_load_2d(to, &map_k, 0, y, full);
      tma_load_2d(to + kObHalf, &map_k, 64, y, full);
    }
    if (lane < 2 * p.nt * p.rep) {
      const int h = lane & 1, r = (lane >> 1) % p.rep, tt = (lane >> 1) / p.rep;
      tma_load_3d(sq + h * q_half + (tt * kObTile + r * p.rp) * 128, &map_q, 64 * h, head * p.nq, b * p.n_obs + tt * p.jt, full);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_d = tmem_slot;
  cl.barrier_arrive();
  grid_dep_launch();  // (not before the tensor memory is ours: a kernel behind that took it first would wait for this one)
  if (bad && rank == 0 && head == 0 && tid == 0) atomicOr(p.status, MC_FLAG_BAD_METADATA);

  // (one thread)
  auto products = [&](int pass, uint32_t done) {
    const uint64_t d0 = smem_desc_k128(0);
    for (int j = 0; j < (T == 1 ? 1 : live); ++j) {
      for (int tt = 0; tt < p.nt; ++tt) {
        const int n_cols = pass == 1 ? kObTile : (min(p.rows - tt * kObTile, kObTile) + 15) / 16 * 16;
        const uint32_t idesc = umma_idesc<DT, 8>() - (1u << 17) + ((uint32_t)(n_cols >> 3) << 17);
        const uint32_t d = tmem_d + ((j << two) + tt + (pass == 2 && both ? units : 0)) * kObTile;
#pragma unroll
        for (int k = 0; k < kHeadDim / 16; ++k) {
          const uint64_t dq = d0 + (uint64_t)((sq + tt * kObHalf + (k >> 2) * q_half) >> 4) + (uint64_t)(2 * (k & 3));
          const uint64_t dk = d0 + (uint64_t)((sk + j * kObTileBytes + (k >> 2) * kObHalf) >> 4) + (uint64_t)(2 * (k & 3));
          if (pass == 1) umma_f16(d, dq, dk, idesc, k > 0 ? 1u : 0u);
          else umma_f16(d, dk, dq, idesc, k > 0 ? 1u : 0u);
        }
      }
    }
    umma_commit(done);
  };
  if (live && warp == 0) {
    if (lane == 0 && mbar_wait_lean(full, 0, s_abort, p.status)) {
      tc_fence_after();
#pragma unroll
      for (int pass = 1; pass <= 2; ++pass)
        if (pass == 1 || both) products(pass, pass == 1 ? done1 : done2);
    }
    __syncwarp();
  }

  // a group's unit: tile j, row tile tt; `shares` groups have the same
  const int grp = warp >> 2, quad = warp & 3, gl = quad * 32 + lane;
  const int unit = grp & (units - 1), j = unit >> two, tt = unit & two, shares = (kObGroups / T) >> two, share = grp / T >> two;
  const int row0 = tt * kObTile, n_rows = min(p.rows - row0, kObTile), tj = t0 + j * kObTile;
  const uint32_t tbuf = tmem_d + ((uint32_t)(quad * 32) << 16);
  const bool no_max = CAP && p.rule.cap_log2 <= 100.f && p.rule.slopes == nullptr;
  const View v0 = ob_view(p, s, max(s.last - p.n_obs + 1, -1)), v1 = ob_view(p, s, s.last);
  const bool easy = !p.positions && !p.rule.slopes && tj + kObTile <= min(n, v0.q_pos + 1) && (tj + kObTile <= v0.prefix || tj >= v1.lo_pos);
  const int at = (page * H + head) * ps + ((t0 + tid) & (ps - 1));  // where the weight of token t0 + tid lives
  if (tid < T * kObTile) {
    int pos = t0 + tid < n ? t0 + tid : kObNoToken;
    if (p.positions && page_ok(p.g, page)) pos = p.positions[at];
    pos_s[tid] = pos;
  }
  if (tid < p.rows) {  // what pass 2 has to know of a row
    const View v = ob_view(p, s, max(s.last - p.n_obs + 1 + (tid >> p.nq_shift), -1));
    qpos_s[tid] = v.q_pos;
    lo_s[tid] = v.lo_pos;
    slope_s[tid] = p.rule.slopes ? p.rule.slopes[head * p.nq + (tid & (p.nq - 1))] * kLog2e : 0.f;
  }
  __syncthreads();

  // ---- pass 1: the lane's query row, a share of the columns that its copy takes
  float m = no_max ? 0.f : -INFINITY, l = 0.f;
  bool good = true;
  if (j < live) {
    good = __all_sync(0xffffffffu, mbar_wait_lean(done1, 0, s_abort, p.status));
    tc_fence_after();
    const int c_lo = gl & ~(p.rp - 1), r_own = gl & (p.rp - 1);
    if (good && ((quad * 32) & (p.rp - 1)) < n_rows) {
      const int r = row0 + min(r_own, n_rows - 1);
      const View vw = {qpos_s[r], s.prefix, lo_s[r]};
      uint64_t lr = 0;
#pragma unroll 1
      for (int ch = c_lo + share * kObChunk; ch < c_lo + p.rp; ch += shares * kObChunk) {
        uint32_t raw[kObChunk];
        tmem_load(tbuf + unit * kObTile + ch, raw);
        add_columns<CAP>(p, raw, easy, pos_s + j * kObTile + ch, vw, slope_s[r], no_max, m, lr);
      }
      float la, lb;
      unpack2(lr, la, lb);
      l = la + lb;
    }
  }
  part_s[grp * kObTile + gl] = make_float2(l == 0.f ? -INFINITY : m, l);
  if (!both) tc_fence_before();
  __syncthreads();
  if (!both && live && tid == 0 && good) {
    tc_fence_after();
    products(2, done2);
  }
  __syncwarp();
  // ---- a row's parts: of the CTA's groups and copies, then of the cluster's CTAs
  cl.barrier_wait();  // (every CTA of the cluster runs: its shared memory may be written)
  if (tid < p.rows) {
    const int row_tile = tid / kObTile, r = tid % kObTile;
    float mm = -INFINITY, ll = 0.f;
    for (int k = 0; k < (kObGroups >> two) * p.rep; ++k) {
      const int g = p.nt == 1 ? k / p.rep : 2 * (k / p.rep) + row_tile;
      const float2 e = part_s[g * kObTile + (k % p.rep) * p.rp + r];
      if (e.y == 0.f) continue;
      const float M = fmaxf(mm, e.x);
      ll = (ll == 0.f ? 0.f : ll * ex2(mm - M)) + e.y * ex2(e.x - M);
      mm = M;
    }
    for (int c = 0; c < C; ++c) *cl.map_shared_rank(all_s + rank * kOsRows + tid, c) = make_float2(mm, ll);
  }
  cl.sync();
  if (tid < p.rows) {
    float mm = -INFINITY, ll = 0.f;
    for (int c = 0; c < C; ++c) {
      const float2 e = all_s[c * kOsRows + tid];
      if (e.y != 0.f) mm = fmaxf(mm, e.x);
    }
    for (int c = 0; c < C; ++c) {
      const float2 e = all_s[c * kOsRows + tid];
      if (e.y != 0.f) ll = fmaf(e.y, ex2(e.x - mm), ll);
    }
    neg_lse[tid] = ll == 0.f ? -INFINITY : -(mm + log2f(ll));  // (a row that saw nothing gives nothing)
  }
  __syncthreads();
  // ---- pass 2: the lane's token, a share of the rows
  float w = 0.f;
  if (j < live) {
    good = __all_sync(0xffffffffu, mbar_wait_lean(done2, 0, s_abort, p.status)) && good;
    tc_fence_after();
    if (good) {
      const int pos = pos_s[j * kObTile + gl];
      uint64_t wa = 0, wb = 0;
#pragma unroll 1
      for (int r0 = share * kObChunk; r0 < n_rows; r0 += shares * kObChunk) {
        uint32_t raw[kObChunk];
        tmem_load(tbuf + (unit + (both ? units : 0)) * kObTile + r0, raw);
        ulonglong2 z2[kObChunk / 4];
#pragma unroll
        for (int k = 0; k < kObChunk / 4; ++k) z2[k] = reinterpret_cast<const ulonglong2*>(neg_lse + row0 + r0)[k];
        const ObRows rows = {neg_lse + row0 + r0, slope_s + row0 + r0, qpos_s + row0 + r0, lo_s + row0 + r0, min(n_rows - r0, kObChunk), s.prefix};
        add_rows<CAP>(p, raw, z2, easy, rows, pos, wa, wb, w);
      }
      float a0, a1, b0, b1;
      unpack2(wa, a0, a1);
      unpack2(wb, b0, b1);
      w += (a0 + a1) + (b0 + b1);
    }
  }
  w_s[grp * kObTile + gl] = w;
  tc_fence_before();
  __syncthreads();
  if (tid < T * kObTile && page_ok(p.g, page)) {
    const int jt = tid / kObTile;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < kObGroups; ++g)
      if ((g & (units - 1)) >> two == jt) sum += w_s[g * kObTile + (tid & (kObTile - 1))];
    p.weights[at] = (p.add ? p.weights[at] : 0.f) + sum;
  }
  if (*s_abort) {  // let copies in flight land before the CTA's memory is released
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
  if (warp == 1) tmem_dealloc(tmem_d, tmem_cols);
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kObMaxCtas = 256;
size_t layer_observe_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int n_obs) {
  const size_t rows = (size_t)n_obs * (cfg->n_q_heads / cfg->n_kv_heads);
  return align_up(((size_t)kObMaxCtas + (size_t)bt->batch * cfg->n_kv_heads) * rows * kObGroups * 2 * sizeof(float), 256);
}

// Tiles per CTA of the one-launch kernel, 0: the two launches.  The fewest with which its clusters run in one wave, a CTA
// per SM.  (Larger clusters fill the GPU's partitions less well: 16 of eight CTAs, and 24 of six, took two waves.)  One
// wave always won: 8 kv heads under 32, 32 queries, 512 tokens 9.7 us against 22.4 (one prompt), 15.3 against 26.8 (eight,
// two tiles each), 24.3 against 29.4 (sixteen, four tiles each); 4096 tokens 23.5 against 29.7; 32 heads, 32 queries, 512
// tokens 8.7 against 14.6 (one prompt), 11.3 against 15.7 (two), 15.1 against 17.8 (four); 64 queries of 8 / 32 heads, 1024
// tokens 15.2 against 24.9 (one prompt), 23.9 against 29.8 (four).
static int short_tiles(int tiles, long long segs, int nt, int n_sm) {
  for (int per = 1; per * nt <= kOsMaxTiles; per *= 2) {
    const int cluster = (tiles + per - 1) / per;
    const int room = cluster <= 2 ? n_sm : cluster <= 4 ? n_sm - n_sm / 8 : n_sm - n_sm / 4;
    if (tiles >= 1 && cluster <= kOsMaxCluster && segs * cluster <= room) return per;
  }
  return 0;
}

// Shared memory of a CTA of the two launches, and of the one.
static constexpr size_t observe_smem(int batch) {
  return 1024 + kObSmem + (2 * kObMaxStages + 4 + 2 * kObGroups) * 8 + 16 + kObGroups * kObTile * (2 * 8 + 8) + (size_t)(batch + 1) * 4 +
         (size_t)batch * sizeof(ObSeq);
}
static constexpr size_t short_smem(int tiles, int nt) { return 1024 + (size_t)(tiles + nt) * kObTileBytes + kOsArrays; }
static_assert(short_smem(1, 2) >= 120 * 1024, "the largest size of a launch");

mc_status launch_layer_observe(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                               const mc_score_opts* opts, const void* q, int n_obs, int flags, void* workspace, cudaStream_t stream) {
  if (bt->batch == 0) return MC_OK;
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  ObserveParams op;
  op.g = g;
  op.rule = make_score_rule(opts);
  op.positions = layer->positions;
  op.weights = layer->weights;
  op.status = layer->status;
  op.part_ml = (float*)workspace;
  op.n_obs = n_obs;
  op.nq = cfg->n_q_heads / cfg->n_kv_heads;
  op.rows = n_obs * op.nq;
  op.nq_shift = op.nq == 1 ? 0 : op.nq == 2 ? 1 : op.nq == 4 ? 2 : 3;
  op.nt = op.rows > kObTile ? 2 : 1;
  op.slots = kObGroups / op.nt;
  op.rp = op.rows > 64 ? 128 : (op.rows > 32 ? 64 : 32);
  op.rep = kObTile / op.rp;
  op.jt = std::min(n_obs, kObTile / op.nq);
  op.stage_shift = op.nt == 1 ? 2 : 1;
  const bool hidden_tiles = opts->window > 0 || opts->doc_start != nullptr || opts->q_pos != nullptr;
  op.zero = !(flags & MC_LAYER_ACCUMULATE) && hidden_tiles;
  op.add = (flags & MC_LAYER_ACCUMULATE) || hidden_tiles;
  const long long max_tiles = (long long)bt->batch * cfg->n_kv_heads * ((bt->max_seq_len + kObTile - 1) / kObTile);
  op.n_ctas = (int)std::max<long long>(1, std::min<long long>(std::min(n_sm, kObMaxCtas), max_tiles));
  if (opts->softcap > 0.f) {
    const double inv = (double)opts->sm_scale / opts->softcap, top = (double)opts->softcap * kLog2e;
    double scale = inv * top;  // of coefficient j: inv^(2 j + 1) * cap * log2(e)
    for (int j = 0; j < 7; ++j, scale *= inv * inv) {
      if (j < 5) op.tiny[j] = (float)(tanh_tiny(j) * scale);
      op.small[j] = (float)(tanh_small(j) * scale);
    }
    // (a polynomial whose coefficients leave binary32's normal range is not used)
    const auto fits = [](float c) { return fabsf(c) > 1e-37f && fabsf(c) < 1e30f; };
    op.tiny_max = fits(op.tiny[0]) && fits(op.tiny[4]) ? (float)(0.5 / fabs(inv)) : -1.f;
    op.small_max = fits(op.small[0]) && fits(op.small[6]) ? (float)(1.0 / fabs(inv)) : -1.f;
    op.poly_max = std::max(op.tiny_max, op.small_max);
  }
  CUtensorMap map_k, map_q;
  const uint64_t rows = (uint64_t)bt->n_pages * cfg->n_kv_heads * cfg->page_size;
  if (mc_status st = make_map(&map_k, cfg->dtype, layer->k_pool, rows, kHeadDim, cfg->page_size)) return st;
  if (mc_status st = make_map3(&map_q, cfg->dtype, q, (uint64_t)bt->batch * n_obs, cfg->n_q_heads, kHeadDim, op.jt, op.nq)) return st;
  const int tiles = (bt->max_seq_len + kObTile - 1) / kObTile;
  const int per = short_tiles(tiles, (long long)bt->batch * cfg->n_kv_heads, op.nt, n_sm), cluster = per ? (tiles + per - 1) / per : 0;
  if (per) {
    op.add = (flags & MC_LAYER_ACCUMULATE) ? 1 : 0;
    using Short = void (*)(const ObserveParams, const CUtensorMap, const CUtensorMap);
    static const Short shorts[2][2][3] = {
        {{layer_observe_short_kernel<MC_F16, false, 1>, layer_observe_short_kernel<MC_F16, false, 2>, layer_observe_short_kernel<MC_F16, false, 4>},
         {layer_observe_short_kernel<MC_F16, true, 1>, layer_observe_short_kernel<MC_F16, true, 2>, layer_observe_short_kernel<MC_F16, true, 4>}},
        {{layer_observe_short_kernel<MC_BF16, false, 1>, layer_observe_short_kernel<MC_BF16, false, 2>, layer_observe_short_kernel<MC_BF16, false, 4>},
         {layer_observe_short_kernel<MC_BF16, true, 1>, layer_observe_short_kernel<MC_BF16, true, 2>, layer_observe_short_kernel<MC_BF16, true, 4>}}};
    const Short kern = shorts[cfg->dtype == MC_F16 ? 0 : 1][opts->softcap > 0.f ? 1 : 0][per >> 1];
    // (more than half an SM's shared memory: two CTAs on one SM might wait for each other's tensor memory)
    const size_t need = std::max<size_t>(short_smem(per, op.nt), 120 * 1024);
    MC_CUDA_CHECK(allow_smem(kern, short_smem(per, per == kOsMaxTiles ? 1 : 2)));
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(bt->batch * cfg->n_kv_heads * cluster));
    lc.blockDim = dim3(kOsThreads);
    lc.dynamicSmemBytes = need;
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
    MC_CUDA_CHECK(cudaLaunchKernelEx(&lc, kern, op, map_k, map_q));
    MC_CUDA_CHECK(cudaGetLastError());
    return MC_OK;
  }
  const size_t smem = observe_smem(bt->batch);
  using Kernel = void (*)(const ObserveParams, const CUtensorMap, const CUtensorMap);
  static const Kernel kernels[2][2][2] = {
      {{layer_observe_kernel<MC_F16, 1, false>, layer_observe_kernel<MC_F16, 1, true>},
       {layer_observe_kernel<MC_F16, 2, false>, layer_observe_kernel<MC_F16, 2, true>}},
      {{layer_observe_kernel<MC_BF16, 1, false>, layer_observe_kernel<MC_BF16, 1, true>},
       {layer_observe_kernel<MC_BF16, 2, false>, layer_observe_kernel<MC_BF16, 2, true>}}};
  for (int pass = 1; pass <= 2; ++pass) {
    const Kernel kern = kernels[cfg->dtype == MC_F16 ? 0 : 1][pass - 1][opts->softcap > 0.f ? 1 : 0];
    MC_CUDA_CHECK(allow_smem(kern, observe_smem(kMaxLayerBatch)));
    MC_CUDA_CHECK(launch_pdl(kern, dim3(op.n_ctas), dim3(kObThreads), smem, stream, op, map_k, map_q));
  }
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
