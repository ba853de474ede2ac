// Single-query decode attention over one uncompressed layer's paged cache: the layers below MiniCache's start layer
// S (Sec. 4.1 merges S .. L-1 only; the others keep their K and V as they are).
//
//   s_i = cap tanh(sm q.k_i / cap) - slope_h (q_pos - p_i)      (cap, slope: optional)
//   out = sum_i softmax(s)_i v_i  over the tokens that the query sees (causal, window, document, prefix)
//
// One pass over the cache with a running maximum and sum.  The token axis is cut into units of 64 tokens (only units
// that hold a visible token are counted); the grid is T teams of S CTAs, a team takes an equal share of the units of
// the batch, its member j takes them for the kv heads j, j + S, ...: the split of mc_attn.cu, for the same reason
// (equal shares whatever the lengths are, neighbouring tiles of a page streamed at about the same time).
// A warp owns a 16-token slice of each of its CTA's units and is a pipeline of its own: it streams the slices' K and V
// rows through its ring of stages with tiled bulk copies (128-byte swizzle; its lane 0 issues them, an mbarrier per
// stage counts the bytes), consumes them itself and writes a partial result of its own for every piece -- the units of
// one (sequence, kv head) in the team's share --, so that no warp ever waits for another.  Scores never leave
// registers: D = K q^T (16 tokens x 8 query rows) becomes the B operand of V^T P by two 8x8 transposes (movmatrix).
// Two stages of 8 KB per warp, 128 KB per SM: a third stage was SLOWER (7b batch 83 -> 88 us, 16 x 8192 grouped 87 ->
// 93): more requests outstanding than the memory serves well.
// Short sequences are not split: a CTA takes one whole and joins its warps' results itself (launch_layer_attn).
// Measured, from a CUDA graph: 83 us on 8 x 4096 tokens of 32 heads (6.45 TB/s: a copy's rate), 87 us on 16 x 8192 of 8 kv
// heads under a cap.
// Where a slice's rows come from is worked out a lane per slice, 32 slices at a time and one window ahead: a
// dependent load takes microseconds while the copies saturate the memory system.
#include <algorithm>

#include "mc_layer.cuh"
#include "mc_layer.h"
#include "mc_kernels.h"
#include "mc_mma.cuh"
#include "mc_pipe.cuh"
#include "mc_tc.cuh"

namespace mc {

constexpr int kLaUnit = 64;    // tokens per unit of work: a slice per warp
constexpr int kLaSlice = 16;   // tokens per stage: one k step of the V contraction, never more than a page
constexpr int kLaWarps = 4;
constexpr int kLaThreads = kLaWarps * 32;
constexpr int kLaStages = 2;
constexpr int kLaStageBytes = 2 * kLaSlice * kRowBytes;  // K rows, V rows: 8 KB
constexpr int kLaCtasPerSm = 2;
constexpr int kLaBoxBytes = kLaSlice * 128;              // one copy: 16 rows x 64 channels

struct LayerAttnParams {
  Geom g;
  ScoreRule rule;
  char* k_pool;
  char* v_pool;
  int32_t* positions;
  float* weights;
  int32_t* status;
  const char* q;
  const char* k_new;
  const char* v_new;
  float* part_o;   // [(team + sequence)][warp][n_q_heads][128]
  float* part_ml;  // [(team + sequence)][warp][n_q_heads][2]
  float* scores;   // [sequence][unit of the sequence][n_kv_heads][kLaUnit][nq], null unless weights are gathered
  float* lse2;     // [batch][n_q_heads] log-sum-exps in log2 units for the weights' kernel
  int seq_units;   // units of the longest sequence
  int nq, n_q_heads;
  int team_size, n_teams;
  int flags;
  int direct;  // 0, or where in shared memory the warps of a CTA join their results: a team has one sequence, all of it
  unsigned short* out;
  float* lse;
};

// A sequence as the call sees it: its view, and the units that hold a visible token: the first `ua`, then those from
// `ub0` on, `u` in all.  (A cache with positions may hold them in any order: every unit counts.)
struct Seq {
  View view;
  int n, n_tot;  // cached tokens; with the step's new one
  int a, lo, hi; // visible indices [0, a) and [lo, hi) (no positions pool)
  int ua, ub0, u;
  bool bad;
};
__device__ __forceinline__ Seq seq_of(const LayerAttnParams& p, int b) {
  Seq s;
  const int raw = __ldcg(p.g.seq_lens + b);  // (from L2: an eviction ahead in the stream may just have written it)
  s.bad = raw < 0 || raw > p.g.max_seq_len;
  s.n = min(max(raw, 0), p.g.max_seq_len);
  s.n_tot = s.n + (p.k_new != nullptr ? 1 : 0);
  s.view = view_at(p.rule, b, max(p.rule.q_pos ? p.rule.q_pos[b] : s.n_tot - 1, -1));
  s.a = s.lo = 0;
  s.hi = s.n_tot;
  s.ua = (s.n_tot + kLaUnit - 1) / kLaUnit;
  s.ub0 = s.ua;
  s.u = s.ua;
  if (p.positions == nullptr) {
    const int end = min(s.n_tot - 1, s.view.q_pos) + 1;  // one past the last index the query may see
    s.a = max(min(end, s.view.prefix), 0);
    s.lo = max(s.view.lo_pos, s.a);
    s.hi = end;
    s.ua = (s.a + kLaUnit - 1) / kLaUnit;
    s.ub0 = s.ua;
    int ub1 = s.ua;
    if (s.hi > s.lo) {
      s.ub0 = max(s.lo / kLaUnit, s.ua);
      ub1 = max((s.hi + kLaUnit - 1) / kLaUnit, s.ub0);
    }
    if (p.flags & MC_LAYER_APPEND) {  // the unit of the appended row counts whether the query sees it or not
      const int un = s.n / kLaUnit;
      if (ub1 <= s.ub0) s.ub0 = ub1 = max(un, s.ua);
      if (ub1 <= un) ub1 = un + 1;
    }
    s.u = s.ua + (ub1 - s.ub0);
  }
  return s;
}

// Exclusive prefix of the sequences' unit counts in shared memory: pre[batch] = all units.  Every thread calls it.
// `keep` (may be null): the sequences themselves.
__device__ __forceinline__ void unit_prefix(const LayerAttnParams& p, int* pre, int n_threads, int& bad, Seq* keep = nullptr) {
  const int tid = threadIdx.x, lane = tid & 31;
  for (int b = tid; b < p.g.batch; b += n_threads) {
    const Seq s = seq_of(p, b);
    bad |= s.bad ? 1 : 0;
    pre[b + 1] = s.u;
    if (keep != nullptr) keep[b] = s;
  }
  __syncthreads();
  if (tid < 32) {
    const int per = (p.g.batch + 31) / 32;
    const int b0 = min(lane * per, p.g.batch), b1 = min(b0 + per, p.g.batch);
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += pre[b + 1];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    int acc = incl - sum;
    for (int b = b0; b < b1; ++b) {
      acc += pre[b + 1];
      pre[b + 1] = acc;
    }
    if (lane == 0) pre[0] = 0;
  }
  __syncthreads();
}

__device__ __forceinline__ int seq_of_unit(const int* pre, int batch, int x) {
  int lo = 0, hi = batch - 1;  // last b with pre[b] <= x
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Teams that get any units: no team's share is empty, so a sequence's pieces are consecutive teams.
__device__ __forceinline__ int live_teams(const LayerAttnParams& p, int n_units) { return min(p.n_teams, max(n_units, 1)); }

// One slice as a lane of the window knows it.
struct Slice {
  int meta;  // flags | sequence << 5 | kv head << 14
  int t0;    // first token
  int x;     // unit: sequence * seq_units + unit of the sequence
  int page;  // raw page id (looked at only when the slice's turn is near)
};
enum { kSlTokens = 1, kSlLoad = 2, kSlFirst = 4, kSlLast = 8, kSlBadSlot = 16 };
static_assert(kMaxLayerBatch <= 512, "nine bits");

__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <int DT>
__global__ void __launch_bounds__(kLaThreads, kLaCtasPerSm)
layer_attn_split_kernel(const __grid_constant__ LayerAttnParams p, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v) {
  // (lengths, block table and score options are the caller's: read before the wait, as in mc_attn.cu)
  grid_dep_launch();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  int* pos_s = reinterpret_cast<int*>(smem + kLaWarps * kLaStages * kLaStageBytes);     // [warps][stages][16]
  uint64_t* bars = reinterpret_cast<uint64_t*>(pos_s + kLaWarps * kLaStages * kLaSlice);  // [warps][stages]
  Seq* seq_s = reinterpret_cast<Seq*>(bars + kLaWarps * kLaStages);                     // [batch]
  int* pre_s = reinterpret_cast<int*>(seq_s + p.g.batch);                               // [batch + 1]
  volatile int* s_abort = pre_s + p.g.batch + 1;
  float* join_o = reinterpret_cast<float*>(smem + p.direct);  // (direct) [warps][query rows][128]
  float* join_ml = join_o + kLaWarps * p.nq * kHeadDim;        // [warps][query rows][2]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = lane >> 2, t4 = lane & 3, colp = 2 * t4;
  const int mi = lane >> 3, mr = lane & 7;
  const int H = p.g.n_kv_heads, nq = p.nq, shift = p.g.page_shift;
  const uint32_t bar0 = smem_u32(bars + warp * kLaStages);
  const uint32_t st0 = smem_u32(smem) + warp * kLaStages * kLaStageBytes;
  const uint32_t pos0 = smem_u32(pos_s + warp * kLaStages * kLaSlice);

  if (tid == 32) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  if (tid == 0) {
    for (int s = 0; s < kLaWarps * kLaStages; ++s) mbar_init(smem_u32(bars + s), 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  int bad = 0;
  unit_prefix(p, pre_s, kLaThreads, bad, seq_s);  // (ends with a barrier)
  const int n_units = pre_s[p.g.batch];
  const int teams = live_teams(p, n_units);
  const int team = blockIdx.x / p.team_size, member = blockIdx.x % p.team_size;
  int x_begin = 0, x_end = 0;
  if (p.direct) {
    x_begin = pre_s[team];
    x_end = pre_s[team + 1];
  } else if (team < teams) {
    x_begin = (int)((long long)n_units * team / teams);
    x_end = (int)((long long)n_units * (team + 1) / teams);
  }
  const int nx = x_end - x_begin;
  const int n_heads = member < H ? (H - member + p.team_size - 1) / p.team_size : 0;
  const int n_slices = nx * n_heads;  // of each warp

  // slice i of this warp: head by head, unit by unit
  auto load_slice = [&](int i) {
    Slice s;
    s.meta = s.t0 = s.x = s.page = 0;
    if (i >= n_slices) return s;
    const int hd = n_heads == 1 ? 0 : i / nx, rem = i - hd * nx;
    const int head = member + hd * p.team_size;
    const int x = x_begin + rem;
    const int b = seq_of_unit(pre_s, p.g.batch, x);
    const Seq& q = seq_s[b];
    const int k = x - pre_s[b];
    s.x = b * p.seq_units + k;
    s.t0 = (k < q.ua ? k : q.ub0 + k - q.ua) * kLaUnit + warp * kLaSlice;
    // (without a positions pool a slice that holds no visible token, nor the row to append, is left out)
    const bool wanted = p.positions != nullptr || s.t0 < q.a || (s.t0 + kLaSlice > q.lo && s.t0 < q.hi) ||
                        ((p.flags & MC_LAYER_APPEND) && q.n >= s.t0 && q.n < s.t0 + kLaSlice);
    int fl = 0;
    if (wanted && s.t0 < q.n_tot) fl |= kSlTokens;
    if (wanted && s.t0 < q.n) fl |= kSlLoad;
    if (x == x_begin || k == 0) fl |= kSlFirst;
    if (x + 1 == x_end || k + 1 == q.u) fl |= kSlLast;
    if ((fl & kSlLoad) || ((fl & kSlTokens) && (p.flags & MC_LAYER_APPEND))) {
      const int slot = s.t0 >> shift;
      if (slot < p.g.max_pages_per_seq) s.page = p.g.block_table[(size_t)b * p.g.max_pages_per_seq + slot];
      else fl |= kSlBadSlot;
    }
    s.meta = fl | b << 5 | head << 14;
    return s;
  };
  // row (of the pools' rows) where a slice begins, -1 if nothing is to be copied; a page id outside the pools reads
  // page 0 and is flagged
  auto slice_row = [&](int page, int head, int t0) {
    if (!page_ok(p.g, page)) page = 0;
    return (page * H + head) * p.g.page_size + (t0 & (p.g.page_size - 1));
  };
  auto row_of = [&](const Slice& s) {
    if (!(s.meta & kSlLoad)) return -1;
    if ((s.meta & kSlBadSlot) || !page_ok(p.g, s.page)) atomicOr(p.status, MC_FLAG_BAD_METADATA);
    return slice_row(s.page, s.meta >> 14, s.t0);
  };
  Slice win = load_slice(lane), nxt = load_slice(32 + lane);

  auto load_q = [&](int b, int head, uint32_t (&q0)[8], uint32_t (&q2)[8]) {
    // B fragment: query row `row`, channels 16 ks + 2 t4 + {0, 1} and + {8, 9}
    const uint32_t* src = reinterpret_cast<const uint32_t*>(p.q) + ((size_t)b * p.n_q_heads + head * nq + row) * (kHeadDim / 2) + t4;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      q0[ks] = row < nq ? src[8 * ks] : 0u;
      q2[ks] = row < nq ? src[8 * ks + 4] : 0u;
    }
  };
  grid_dep_wait();
  if (bad) atomicOr(p.status, MC_FLAG_BAD_METADATA);

  int win_row = row_of(win), nxt_row = -1;
  auto issue = [&](int i) {  // slice i into its stage (four lanes issuing a box each were slower than one lane issuing four)
    if (i >= n_slices) return;
    // (i lies in the current window or, at its end, in the next one)
    const int y = __shfl_sync(0xffffffffu, i >= 32 && (i & 31) < kLaStages - 1 ? nxt_row : win_row, i & 31);
    if (y < 0 || *s_abort) return;
    const int s = i % kLaStages;
    const uint32_t bar = bar0 + 8 * s;
    if (lane == 0) {
      const uint32_t dst = st0 + s * kLaStageBytes;
      mbar_expect_tx(bar, (uint32_t)(kLaStageBytes + (p.positions ? kLaSlice * 4 : 0)));
      tma_load_2d(dst, &map_k, 0, y, bar);
      tma_load_2d(dst + kLaBoxBytes, &map_k, 64, y, bar);
      tma_load_2d(dst + 2 * kLaBoxBytes, &map_v, 0, y, bar);
      tma_load_2d(dst + 3 * kLaBoxBytes, &map_v, 64, y, bar);
      if (p.positions) bulk_load(pos0 + s * kLaSlice * 4, p.positions + y, kLaSlice * 4, bar);
    }
  };
  for (int i = 0; i < kLaStages - 1; ++i) issue(i);
  // (behind the wait: the queries may be what the kernel ahead wrote, another layer's output for instance)
  uint32_t q0[8], q2[8];
  {
    const int meta = __shfl_sync(0xffffffffu, win.meta, 0);
    if (n_slices > 0) load_q((meta >> 5) & 511, meta >> 14, q0, q2);
  }

  if (p.direct && nx == 0) {  // no token at all
    for (int hd = 0; hd < n_heads; ++hd) {
      const size_t orow = (size_t)team * p.n_q_heads + (member + hd * p.team_size) * nq;
      for (int i = tid; i < nq * 16; i += kLaThreads) reinterpret_cast<uint4*>(p.out + orow * kHeadDim)[i] = make_uint4(0u, 0u, 0u, 0u);
      if (tid < nq) {
        if (p.lse != nullptr) p.lse[orow + tid] = -INFINITY;
        if (p.scores != nullptr) p.lse2[orow + tid] = INFINITY;
      }
    }
  }

  float acc[8][4];
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;  // query rows colp, colp + 1
  float sl0 = 0.f, sl1 = 0.f;
  Seq sq = {};
  uint32_t phase = 0;  // bit s: parity of stage s's next completion

  for (int i = 0; i < n_slices; ++i) {
    const int src = i & 31;
    if (src == 0 && i > 0) {
      win = nxt;
      win_row = nxt_row;
      nxt = load_slice((i & ~31) + 32 + lane);
    }
    if (src == 32 - kLaStages) nxt_row = row_of(nxt);  // (its loads are long done)
    // the stage of the slice before this one is free: its warp has read it
    __syncwarp();
    issue(i + kLaStages - 1);
    const int fl = __shfl_sync(0xffffffffu, win.meta, src);  // (flags in the low bits)
    const int b = (fl >> 5) & 511, head = fl >> 14;
    const int t0 = __shfl_sync(0xffffffffu, win.t0, src);
    const int s = i % kLaStages;
    if (fl & kSlFirst) {
      m0 = m1 = -INFINITY;
      l0 = l1 = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[j][k] = 0.f;
      sq = seq_s[b];
      // what this piece will read late and the next piece first goes to L1 meanwhile (a demand load takes microseconds
      // behind the stream): the step's new rows, the next piece's queries
      if (p.k_new && lane < 4) {
        const char* r = ((lane & 2) ? p.v_new : p.k_new) + ((size_t)b * H + head) * kRowBytes + (lane & 1) * 128;
        asm volatile("prefetch.global.L1 [%0];" ::"l"(r));
      }
      const uint32_t later = __ballot_sync(0xffffffffu, (win.meta & kSlFirst) != 0) & ~((2u << src) - 1u);
      if (later) {
        const int mn = __shfl_sync(0xffffffffu, win.meta, __ffs(later) - 1);
        if (lane < 2 * nq)
          asm volatile("prefetch.global.L1 [%0];" ::"l"(p.q + (((size_t)((mn >> 5) & 511) * p.n_q_heads + (mn >> 14) * nq) * kRowBytes) + lane * 128));
      }
      if (p.rule.slopes) {
        sl0 = colp < nq ? p.rule.slopes[head * nq + colp] * kLog2e : 0.f;
        sl1 = colp + 1 < nq ? p.rule.slopes[head * nq + colp + 1] * kLog2e : 0.f;
      }
    }
    if (fl & kSlTokens) {
      const uint32_t sb = st0 + s * kLaStageBytes;
      const bool has_new = p.k_new != nullptr && sq.n >= t0 && sq.n < t0 + kLaSlice;  // (warp-uniform)
      uint4 rown = make_uint4(0u, 0u, 0u, 0u);
      if (has_new) {  // lanes 0..15: the new K row's chunks, 16..31: the V row's
        const char* src_row = (lane < 16 ? p.k_new : p.v_new) + ((size_t)b * H + head) * kRowBytes;
        rown = *reinterpret_cast<const uint4*>(src_row + (lane & 15) * 16);
      }
      if (fl & kSlLoad) {
        mbar_wait(bar0 + 8 * s, (phase >> s) & 1, s_abort, p.status);  // (on a time-out the CTA only runs to its end)
        phase ^= 1u << s;
      }
      bool wrote = false;
      if (has_new) {
        // the step's row takes its place in the stage (its slot of the page holds nothing yet) and, on request, in the cache
        const int r = sq.n - t0, c = lane & 15;
        const uint32_t a = sb + (lane < 16 ? 0 : 2 * kLaBoxBytes) + (c >> 3) * kLaBoxBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(rown.x), "r"(rown.y), "r"(rown.z), "r"(rown.w) : "memory");
        wrote = true;
        if (p.positions && lane == 0) pos_s[(warp * kLaStages + s) * kLaSlice + r] = sq.view.q_pos;
        if (p.flags & MC_LAYER_APPEND) {
          const int page = __shfl_sync(0xffffffffu, win.page, src);
          if (!(fl & kSlBadSlot) && page_ok(p.g, page)) {
            const size_t at = (size_t)slice_row(page, head, t0) + r;
            *reinterpret_cast<uint4*>((lane < 16 ? p.k_pool : p.v_pool) + at * kRowBytes + c * 16) = rown;
            if (p.positions && lane == 0) p.positions[at] = sq.view.q_pos;
            if (p.weights && !(p.flags & MC_LAYER_ACCUMULATE) && lane == 0) p.weights[at] = 0.f;
          } else if (lane == 0) {
            atomicOr(p.status, MC_FLAG_BAD_METADATA);
          }
        }
        __syncwarp();
      }
      // ---- scores: D[token][query row], k steps in four chains
      float d[4][4] = {};  // four chains of k steps
      {
        const int tr = (mi & 1) * 8 + mr;
        uint32_t ra[8][4];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const int c = 2 * ks + (mi >> 1);
          ldsm_x4(sb + (c >> 3) * kLaBoxBytes + tr * 128 + (((c & 7) ^ mr) << 4), ra[ks][0], ra[ks][1], ra[ks][2], ra[ks][3]);
        }
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) mma_rows<DT>(d[ks & 3], ra[ks][0], ra[ks][1], ra[ks][2], ra[ks][3], q0[ks], q2[ks]);
      }
      float sc[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) sc[k] = (d[0][k] + d[1][k]) + (d[2][k] + d[3][k]);
      // ---- masks (tokens t0 + row and + 8), the scores' form, the distance bias
      uint32_t hidden = 0;  // bit r: token t0 + r is not seen (the same in every lane)
      {
        int p0 = t0 + row, p8 = p0 + 8;
        bool v0 = true, v8 = true, whole;
        if (p.positions) {
          const int* ps = pos_s + (warp * kLaStages + s) * kLaSlice;
          v0 = p0 < sq.n_tot;
          v8 = p8 < sq.n_tot;
          p0 = ps[row];
          p8 = ps[row + 8];
          v0 = v0 && sq.view.sees(p0);
          v8 = v8 && sq.view.sees(p8);
          whole = __all_sync(0xffffffffu, v0 && v8);
        } else {
          whole = (t0 + kLaSlice <= sq.a) || (t0 >= sq.lo && t0 + kLaSlice <= sq.hi);
          if (!whole) {
            v0 = p0 < sq.a || (p0 >= sq.lo && p0 < sq.hi);
            v8 = p8 < sq.a || (p8 >= sq.lo && p8 < sq.hi);
          }
        }
        // (a row that is not seen, stale or poisoned, has no say in which form of the cap the others take)
        if (!whole && p.rule.cap_log2 > 0.f) {
          if (!v0) sc[0] = sc[1] = 0.f;
          if (!v8) sc[2] = sc[3] = 0.f;
        }
        scores_of(p.rule, sc);
        if (p.rule.slopes) {
          const float e0 = (float)(sq.view.q_pos - p0), e8 = (float)(sq.view.q_pos - p8);
          sc[0] = fmaf(-sl0, e0, sc[0]);
          sc[1] = fmaf(-sl1, e0, sc[1]);
          sc[2] = fmaf(-sl0, e8, sc[2]);
          sc[3] = fmaf(-sl1, e8, sc[3]);
        }
        if (!whole) {
          if (!v0) sc[0] = sc[1] = -INFINITY;
          if (!v8) sc[2] = sc[3] = -INFINITY;
          const uint32_t h0 = __ballot_sync(0xffffffffu, !v0), h8 = __ballot_sync(0xffffffffu, !v8);
#pragma unroll
          for (int r = 0; r < 8; ++r) hidden |= ((h0 >> (4 * r)) & 1u) << r | ((h8 >> (4 * r)) & 1u) << (r + 8);
        }
      }
      if (p.scores != nullptr) {
        const int x = __shfl_sync(0xffffffffu, win.x, src);
        float* o = p.scores + (((size_t)x * H + head) * kLaUnit + (t0 & (kLaUnit - 1)) + row) * nq + colp;
        if (nq == 1) {
          if (t4 == 0) {
            o[0] = sc[0];
            o[8] = sc[2];
          }
        } else if (colp < nq) {
          *reinterpret_cast<float2*>(o) = make_float2(sc[0], sc[1]);
          *reinterpret_cast<float2*>(o + 8 * nq) = make_float2(sc[2], sc[3]);
        }
      }
      if (hidden != 0xffffu) {
        // ---- running maximum and sum (the lanes compare notes only when one of them holds a larger score)
        float n0 = fmaxf(sc[0], sc[2]), n1 = fmaxf(sc[1], sc[3]);
        if (__any_sync(0xffffffffu, n0 > m0 || n1 > m1)) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, o));
            n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
          }
          n0 = fmaxf(n0, m0);
          n1 = fmaxf(n1, m1);
          const float f0 = n0 == m0 ? 1.f : ex2(m0 - n0), f1 = n1 == m1 ? 1.f : ex2(m1 - n1);
          m0 = n0;
          m1 = n1;
          l0 *= f0;
          l1 *= f1;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            acc[j][0] *= f0;
            acc[j][1] *= f1;
            acc[j][2] *= f0;
            acc[j][3] *= f1;
          }
        }
        // (a row that has seen nothing yet has maximum -inf: its probabilities are 2^-inf, not NaN)
        const float b0 = m0 == -INFINITY ? 0.f : m0, b1 = m1 == -INFINITY ? 0.f : m1;
        const float e0 = ex2(sc[0] - b0), e1 = ex2(sc[1] - b1), e2 = ex2(sc[2] - b0), e3 = ex2(sc[3] - b1);
        l0 += e0 + e2;
        l1 += e1 + e3;
        // P as the B operand: rounded once to the storage type (half a step of a number <= 1, as a V element carries)
        const uint32_t pb0 = transpose8(Elem<DT>::pack(e0, e1)), pb1 = transpose8(Elem<DT>::pack(e2, e3));
        if (hidden) {  // rows that are not seen may hold anything, infinities and NaN too: 0 * x has to stay 0
          for (int k = lane; k < kLaSlice * 16; k += 32) {
            const int r = k >> 4, c = k & 15;
            if ((hidden >> r) & 1u)
              asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(sb + 2 * kLaBoxBytes + (c >> 3) * kLaBoxBytes + r * 128 +
                                                                         ((c & 7) << 4)),
                           "r"(0u)
                           : "memory");
          }
          wrote = true;
          __syncwarp();
        }
        // ---- V^T P: D[channel][query row]
        const int tr = (mi >> 1) * 8 + mr;
        uint32_t ra[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = 2 * j + (mi & 1);
          ldsm_x4_t(sb + 2 * kLaBoxBytes + (c >> 3) * kLaBoxBytes + tr * 128 + (((c & 7) ^ mr) << 4), ra[j][0], ra[j][1], ra[j][2],
                    ra[j][3]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) mma_rows<DT>(acc[j], ra[j][0], ra[j][1], ra[j][2], ra[j][3], pb0, pb1);
      }
      if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (fl & kSlLast) {
      if (i + 1 < n_slices) {
        const bool nw = src == 31;
        const int mn = __shfl_sync(0xffffffffu, nw ? nxt.meta : win.meta, (i + 1) & 31);
        load_q((mn >> 5) & 511, mn >> 14, q0, q2);
      }
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, o);
        l1 += __shfl_xor_sync(0xffffffffu, l1, o);
      }
      const size_t prow = ((size_t)(team + b) * kLaWarps + warp) * p.n_q_heads + head * nq;
      float* to = p.direct ? join_o + warp * nq * kHeadDim : p.part_o + prow * kHeadDim;
      float* to_ml = p.direct ? join_ml + warp * nq * 2 : p.part_ml + 2 * prow;
      if (colp < nq) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          to[colp * kHeadDim + 16 * j + row] = acc[j][0];
          to[colp * kHeadDim + 16 * j + row + 8] = acc[j][2];
        }
        if (row == 0) *reinterpret_cast<float2*>(to_ml + 2 * colp) = make_float2(m0, l0);
      }
      if (colp + 1 < nq) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          to[(colp + 1) * kHeadDim + 16 * j + row] = acc[j][1];
          to[(colp + 1) * kHeadDim + 16 * j + row + 8] = acc[j][3];
        }
        if (row == 0) *reinterpret_cast<float2*>(to_ml + 2 * (colp + 1)) = make_float2(m1, l1);
      }
      if (p.direct) {  // the four warps' results, joined as the combine kernel does it
        __syncthreads();
        for (int k = tid; k < nq * 32; k += kLaThreads) {
          const int r = k >> 5, c4 = (k & 31) * 4;
          float M = -INFINITY, L = 0.f;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kLaWarps; ++w) M = fmaxf(M, join_ml[(w * nq + r) * 2]);
#pragma unroll
          for (int w = 0; w < kLaWarps; ++w) {
            const float2 ml = *reinterpret_cast<const float2*>(join_ml + (w * nq + r) * 2);
            const float4 v = *reinterpret_cast<const float4*>(join_o + (w * nq + r) * kHeadDim + c4);
            const float f = ml.y == 0.f ? 0.f : ex2(ml.x - M);
            L = fmaf(f, ml.y, L);
            o.x = fmaf(f, v.x, o.x);
            o.y = fmaf(f, v.y, o.y);
            o.z = fmaf(f, v.z, o.z);
            o.w = fmaf(f, v.w, o.w);
          }
          const float inv = L == 0.f ? 0.f : 1.f / L;
          const size_t orow = (size_t)b * p.n_q_heads + head * nq + r;
          uint2 packed;
          packed.x = Elem<DT>::pack(o.x * inv, o.y * inv);
          packed.y = Elem<DT>::pack(o.z * inv, o.w * inv);
          *reinterpret_cast<uint2*>(p.out + orow * kHeadDim + c4) = packed;
          if (c4 == 0) {
            const float z = L == 0.f ? -INFINITY : M + log2f(L);
            if (p.lse != nullptr) p.lse[orow] = z * kLn2;
            if (p.scores != nullptr) p.lse2[orow] = L == 0.f ? INFINITY : z;
          }
        }
        __syncthreads();  // (before the next head's results take the same place)
      }
    }
  }
  if (*s_abort) {  // let copies in flight land before the CTA's memory is released
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
}

// Joins a sequence's pieces (consecutive teams, a part per warp of their CTAs):
// out = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j.  A block has R query heads, 8 / R warps each: about three parts per
// warp, so that a warp's loads travel together.
constexpr int kLcThreads = 256;
constexpr int kLcWarps = kLcThreads / 32;

template <int DT, int R>
__global__ void __launch_bounds__(kLcThreads) layer_attn_combine_kernel(const __grid_constant__ LayerAttnParams p, unsigned short* out,
                                                                        float* lse) {
  grid_dep_launch();
  __shared__ int pre_s[kMaxLayerBatch + 1];
  __shared__ float4 acc_s[kLcWarps][32];
  __shared__ float red_s[kLcWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.y;
  int bad = 0;
  unit_prefix(p, pre_s, kLcThreads, bad);
  const long long U = pre_s[p.g.batch];
  const int T = live_teams(p, (int)U);
  const int x0 = pre_s[b], u = pre_s[b + 1] - x0;
  // the team of unit x is the last c with floor(U c / T) <= x
  const int c0 = u > 0 ? (int)(((long long)(x0 + 1) * T - 1) / U) : 0;
  const int c1 = u > 0 ? (int)(((long long)(x0 + u) * T - 1) / U) : -1;
  constexpr int GP = kLcWarps / R;  // warps per output row
  const int grp = warp % GP;
  const int hq = blockIdx.x * R + warp / GP;
  const bool active = hq < p.n_q_heads;
  grid_dep_wait();
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (active) {
    const int c_end = (c1 + 1) * kLaWarps;  // (a piece has a part of each of its CTA's warps)
    for (int c = c0 * kLaWarps + grp; c < c_end; c += 4 * GP) {  // four parts in flight
      float2 ml[4];
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c + k * GP < c_end) {
          const size_t prow = (size_t)(c + k * GP + b * kLaWarps) * p.n_q_heads + hq;
          ml[k] = *reinterpret_cast<const float2*>(p.part_ml + 2 * prow);
          v[k] = *reinterpret_cast<const float4*>(p.part_o + prow * kHeadDim + 4 * lane);
        }
      }
      float M2 = M;
#pragma unroll
      for (int k = 0; k < 4; ++k) M2 = fmaxf(M2, ml[k].x);
      const float f = L == 0.f ? 0.f : ex2(M - M2);
      M = M2;
      L *= f;
      o.x *= f;
      o.y *= f;
      o.z *= f;
      o.w *= f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = ml[k].y == 0.f ? 0.f : ex2(ml[k].x - M);
        L = fmaf(w, ml[k].y, L);
        o.x = fmaf(w, v[k].x, o.x);
        o.y = fmaf(w, v[k].y, o.y);
        o.z = fmaf(w, v[k].z, o.z);
        o.w = fmaf(w, v[k].w, o.w);
      }
    }
  }
  if (GP > 1) {
    __shared__ float max_s[kLcWarps];
    acc_s[warp][lane] = o;
    if (lane == 0) {
      red_s[warp] = L;
      max_s[warp] = M;
    }
    __syncthreads();
    if (grp != 0 || !active) return;
    float Ma = M;
    for (int g = 1; g < GP; ++g) Ma = fmaxf(Ma, max_s[warp + g]);
    const float f = L == 0.f ? 0.f : ex2(M - Ma);
    L *= f;
    o.x *= f;
    o.y *= f;
    o.z *= f;
    o.w *= f;
    for (int g = 1; g < GP; ++g) {
      const float lg = red_s[warp + g], fg = lg == 0.f ? 0.f : ex2(max_s[warp + g] - Ma);
      const float4 t = acc_s[warp + g][lane];
      L = fmaf(fg, lg, L);
      o.x = fmaf(fg, t.x, o.x);
      o.y = fmaf(fg, t.y, o.y);
      o.z = fmaf(fg, t.z, o.z);
      o.w = fmaf(fg, t.w, o.w);
    }
    M = Ma;
  } else if (!active) {
    return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;  // (a query that sees nothing: zeros, log-sum-exp -inf)
  const size_t orow = (size_t)b * p.n_q_heads + hq;
  uint2 packed;
  packed.x = Elem<DT>::pack(o.x * inv, o.y * inv);
  packed.y = Elem<DT>::pack(o.z * inv, o.w * inv);
  *reinterpret_cast<uint2*>(out + orow * kHeadDim + lane * 4) = packed;
  if (lane == 0) {
    const float z = L == 0.f ? -INFINITY : M + log2f(L);
    if (lse != nullptr) lse[orow] = z * kLn2;
    if (p.scores != nullptr) p.lse2[orow] = L == 0.f ? INFINITY : z;  // (a row that saw nothing gives no weight)
  }
}

// w_i += sum over the head group of 2^(s_i - lse), from the scores the split kernel left: a block has 1024 tokens of one
// kv head, a thread four of them.  Where their weights live follows from the caller's tables (before the wait); scores,
// old weights and log-sum-exps are then requested together.  (Inside the combine kernel, each block joining the partial
// sums for itself, this took 19 us on 4 x 32768 tokens.)
constexpr int kLwTokens = 1024;

template <int NQ>
__global__ void __launch_bounds__(kLcThreads) layer_attn_weights_kernel(const __grid_constant__ LayerAttnParams p, int blocks) {
  grid_dep_launch();
  const int tid = threadIdx.x, b = blockIdx.y, head = blockIdx.x / blocks;
  const Seq sq = seq_of(p, b);
  constexpr int kOwn = kLwTokens / kLcThreads, kStep = kLwTokens / kLaUnit;
  // (the grid is sized for the GPU, not for the longest length a sequence might have: a block takes every `blocks`-th chunk)
  bool waited = false;
  for (int k0 = (blockIdx.x % blocks) * kStep; k0 < sq.u; k0 += blocks * kStep) {
    int at[kOwn];
    long long from[kOwn];  // (past 32 bits in a long batch)
    bool fresh[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = tid + j * kLcThreads, k = k0 + i / kLaUnit, in = i % kLaUnit;
      const int t = (k < sq.ua ? k : sq.ub0 + k - sq.ua) * kLaUnit + in, slot = t >> p.g.page_shift;
      fresh[j] = t == sq.n;  // the appended row: its weight begins here
      at[j] = -1;
      from[j] = -1;
      if (k >= sq.u || t >= sq.n_tot || slot >= p.g.max_pages_per_seq || (fresh[j] && !(p.flags & MC_LAYER_APPEND))) continue;
      const bool seen = p.positions != nullptr || t < sq.a || (t >= sq.lo && t < sq.hi);
      if (!seen && !fresh[j]) continue;  // (no score was written)
      const int page = p.g.block_table[(size_t)b * p.g.max_pages_per_seq + slot];
      if (!page_ok(p.g, page)) continue;  // (flagged by the split kernel)
      at[j] = (page * p.g.n_kv_heads + head) * p.g.page_size + (t & (p.g.page_size - 1));
      if (seen) from[j] = ((long long)(b * p.seq_units + k) * p.g.n_kv_heads + head) * kLaUnit + in;
    }
    if (!waited) grid_dep_wait();
    waited = true;
    float s[kOwn][NQ], w[kOwn], z[NQ];
#pragma unroll
    for (int r = 0; r < NQ; ++r) z[r] = p.lse2[(size_t)b * p.n_q_heads + head * NQ + r];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      w[j] = at[j] >= 0 && !fresh[j] ? p.weights[at[j]] : 0.f;
      const float* src = p.scores + (size_t)max(from[j], 0LL) * NQ;
      if (NQ % 4 == 0) {
#pragma unroll
        for (int r = 0; r < NQ; r += 4) {
          const float4 v = from[j] >= 0 ? *reinterpret_cast<const float4*>(src + r) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
          s[j][r] = v.x;
          s[j][(r + 1) % NQ] = v.y;
          s[j][(r + 2) % NQ] = v.z;
          s[j][(r + 3) % NQ] = v.w;
        }
      } else {
#pragma unroll
        for (int r = 0; r < NQ; ++r) s[j][r] = from[j] >= 0 ? src[r] : -INFINITY;
      }
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (at[j] < 0) continue;
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < NQ; ++r) sum += s[j][r] == -INFINITY ? 0.f : ex2(s[j][r] - z[r]);  // (a row not seen: nothing, whatever z)
      p.weights[at[j]] = w[j] + sum;
    }
  }
  if (!waited) grid_dep_wait();  // (a grid that ended without it would let the kernel behind overtake those ahead)
}

// ---- host side ------------------------------------------------------------------------------------
struct LayerAttnPlan {
  int team_size, n_teams;
  long long max_units;  // of the batch
  int seq_units;        // of the longest sequence
  size_t o_bytes, ml_bytes, score_bytes, lse_bytes;
};
// n_sm: multiprocessors of the device; the workspace is sized for kLaMaxCtas / kLaCtasPerSm of them, so that its size
// needs no device.
constexpr int kLaMaxCtas = 512;
static LayerAttnPlan layer_attn_plan(const mc_config* cfg, const mc_batch* bt, int flags, int n_sm) {
  LayerAttnPlan pl;
  const int slots = std::min(n_sm * kLaCtasPerSm, kLaMaxCtas);
  const int per_cta = (cfg->n_kv_heads + std::min(slots, 32) - 1) / std::min(slots, 32);
  pl.team_size = (cfg->n_kv_heads + per_cta - 1) / per_cta;
  pl.seq_units = bt->max_seq_len / kLaUnit + 1;  // (with the step's new token)
  pl.max_units = (long long)bt->batch * pl.seq_units;
  pl.n_teams = (int)std::max<long long>(1, std::min<long long>(slots / pl.team_size, pl.max_units));
  const size_t prow = (size_t)(pl.n_teams + bt->batch) * kLaWarps * cfg->n_q_heads;
  pl.o_bytes = align_up(prow * kHeadDim * 4, 256);
  pl.ml_bytes = align_up(prow * 2 * 4, 256);
  pl.score_bytes = (flags & MC_LAYER_ACCUMULATE) ? align_up((size_t)pl.max_units * kLaUnit * cfg->n_q_heads * 4, 256) : 0;
  pl.lse_bytes = (flags & MC_LAYER_ACCUMULATE) ? align_up((size_t)bt->batch * cfg->n_q_heads * 4, 256) : 0;
  return pl;
}
// Shared memory of a CTA: stages, positions, barriers and the batch; where its warps join their results.
static constexpr size_t attn_smem_used(int batch) {
  return ((size_t)kLaWarps * kLaStages * (kLaStageBytes + kLaSlice * 4 + 8) + (size_t)(batch + 2) * (4 + sizeof(Seq)) + 15) / 16 * 16;
}
static constexpr size_t attn_smem_join(int nq) { return (size_t)kLaWarps * nq * (kHeadDim + 2) * 4; }
static_assert(1024 + attn_smem_used(kMaxLayerBatch) + attn_smem_join(8) >= 80 * 1024, "the largest size of a launch");

size_t layer_attn_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int flags) {
  const LayerAttnPlan pl = layer_attn_plan(cfg, bt, flags, kLaMaxCtas / kLaCtasPerSm);
  return pl.o_bytes + pl.ml_bytes + pl.score_bytes + pl.lse_bytes;
}

mc_status launch_layer_attn(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_cache* layer,
                            const mc_score_opts* opts, const void* q, const void* k_new, const void* v_new, int flags, void* out,
                            float* lse, void* workspace, cudaStream_t stream) {
  if (bt->batch == 0) return MC_OK;
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  const LayerAttnPlan pl = layer_attn_plan(cfg, bt, flags, n_sm);
  CUtensorMap map_k, map_v;
  const uint64_t rows = (uint64_t)std::max<int64_t>(bt->n_pages, 1) * cfg->n_kv_heads * cfg->page_size;
  if (mc_status st = make_map(&map_k, cfg->dtype, layer->k_pool, rows, kHeadDim, kLaSlice)) return st;
  if (mc_status st = make_map(&map_v, cfg->dtype, layer->v_pool, rows, kHeadDim, kLaSlice)) return st;
  LayerAttnParams ap;
  ap.g = g;
  ap.rule = make_score_rule(opts);
  ap.k_pool = (char*)layer->k_pool;
  ap.v_pool = (char*)layer->v_pool;
  ap.positions = layer->positions;
  ap.weights = layer->weights;
  ap.status = layer->status;
  ap.q = (const char*)q;
  ap.k_new = (const char*)k_new;
  ap.v_new = (const char*)v_new;
  ap.part_o = (float*)workspace;
  ap.part_ml = (float*)((char*)workspace + pl.o_bytes);
  ap.scores = (flags & MC_LAYER_ACCUMULATE) ? (float*)((char*)workspace + pl.o_bytes + pl.ml_bytes) : nullptr;
  ap.lse2 = (float*)((char*)workspace + pl.o_bytes + pl.ml_bytes + pl.score_bytes);
  ap.seq_units = pl.seq_units;
  ap.nq = cfg->n_q_heads / cfg->n_kv_heads;
  ap.n_q_heads = cfg->n_q_heads;
  ap.team_size = pl.team_size;
  ap.flags = flags;
  ap.out = (unsigned short*)out;
  ap.lse = lse;
  // Short sequences, one CTA (team member) for all of each: it writes the output itself and there is no second launch.
  // That costs 2.2 us and 1.1 us per unit of the longest sequence, the split 3.9 us and 1.1 us per unit of a CTA's equal
  // share (32 heads: one sequence of 33 tokens 3.3 against 4.9 us, of 127 4.6 against 5.2, of 255 6.8 against 4.9; nine of
  // 255 8.3 against 10.1).  At most four units, as the lengths behind the bound may differ.
  const long long slots = n_sm * kLaCtasPerSm, ctas = (long long)bt->batch * pl.team_size;
  const bool direct = ctas <= slots && pl.seq_units <= 4 && 2 * (pl.seq_units * slots - std::max(slots, ctas * pl.seq_units)) <= 3 * slots;
  ap.n_teams = direct ? bt->batch : pl.n_teams;
  // (asked for so much that two CTAs fill an SM: with room for a third, an early start behind another kernel packs some
  // SMs with three and leaves others with one -- 83 -> 86 us on 8 x 4096)
  ap.direct = direct ? (int)attn_smem_used(bt->batch) : 0;
  const size_t smem = std::max<size_t>(80 * 1024, 1024 + attn_smem_used(bt->batch) + (direct ? attn_smem_join(ap.nq) : 0));
  auto* split = cfg->dtype == MC_F16 ? layer_attn_split_kernel<MC_F16> : layer_attn_split_kernel<MC_BF16>;
  MC_CUDA_CHECK(allow_smem(split, 1024 + attn_smem_used(kMaxLayerBatch) + attn_smem_join(8)));
  MC_CUDA_CHECK(launch_pdl(split, dim3(ap.n_teams * pl.team_size), dim3(kLaThreads), smem, stream, ap, map_k, map_v));
  if (!direct) {
    // warps per output row: about three parts each
    const long long parts = (long long)kLaWarps * (pl.n_teams / bt->batch + 1);
    int per_block = kLcWarps;  // rows
    while (per_block > 1 && parts > 3 * (kLcWarps / per_block)) per_block /= 2;
    using Combine = void (*)(const LayerAttnParams, unsigned short*, float*);
    static const Combine combines[2][4] = {
        {layer_attn_combine_kernel<MC_F16, 1>, layer_attn_combine_kernel<MC_F16, 2>, layer_attn_combine_kernel<MC_F16, 4>,
         layer_attn_combine_kernel<MC_F16, 8>},
        {layer_attn_combine_kernel<MC_BF16, 1>, layer_attn_combine_kernel<MC_BF16, 2>, layer_attn_combine_kernel<MC_BF16, 4>,
         layer_attn_combine_kernel<MC_BF16, 8>}};
    const Combine combine = combines[cfg->dtype == MC_F16 ? 0 : 1][per_block == 1 ? 0 : per_block == 2 ? 1 : per_block == 4 ? 2 : 3];
    MC_CUDA_CHECK(launch_pdl(combine, dim3((cfg->n_q_heads + per_block - 1) / per_block, bt->batch), dim3(kLcThreads), 0, stream, ap,
                             (unsigned short*)out, lse));
  }
  if (flags & MC_LAYER_ACCUMULATE) {
    const int chunks = (pl.seq_units * kLaUnit + kLwTokens - 1) / kLwTokens, segs = bt->batch * cfg->n_kv_heads;
    const int blocks = std::min(chunks, (8 * n_sm + segs - 1) / segs);  // per (sequence, kv head)
    auto* weights = ap.nq == 1   ? layer_attn_weights_kernel<1>
                    : ap.nq == 2 ? layer_attn_weights_kernel<2>
                    : ap.nq == 4 ? layer_attn_weights_kernel<4>
                                 : layer_attn_weights_kernel<8>;
    MC_CUDA_CHECK(launch_pdl(weights, dim3(cfg->n_kv_heads * blocks, bt->batch), dim3(kLcThreads), 0, stream, ap, blocks));
  }
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
