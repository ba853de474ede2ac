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
// One persistent CTA per SM; the tiles of all (sequence, kv head) segments are shared out equally.  Warp 0 streams K
// tiles (a tiled copy per page and 64-channel half) and the segments' Q; warp 1 issues tcgen05.mma into two
// tensor-memory buffers; two groups of four warps take the tiles in turn, each from its own buffer.  The exponentials
// bound it: 2 R per token, 16 a clock and SM.  Every wait is bounded; tensor memory is released on every path.
#include <algorithm>

#include "mc_layer.cuh"
#include "mc_layer.h"
#include "mc_kernels.h"
#include "mc_pipe.cuh"
#include "mc_tc.cuh"

namespace mc {

constexpr int kObTile = 128;                             // tokens per tile
constexpr int kObHalf = kObTile * 128;                   // bytes of a tile's 64-channel half
constexpr int kObTileBytes = 2 * kObHalf;                // 32 KB
constexpr int kObMaxRows = 256;
constexpr int kObThreads = 320;                          // producer, tensor-core issue, two groups of four warps
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
  float* part_ml;  // [(CTA + segment)][2 groups][rows][2]
  int n_obs, nq, n_q_heads;
  int rows;      // n_obs * nq
  int nt;        // row tiles of 128: 1 or 2
  int rp, rep;   // rows of a copy (32, 64 or 128), copies in a row tile
  int jt;        // queries per Q copy
  int stages;    // K ring
  int add;       // pass 2 adds to the weights (else it writes them)
  int zero;      // pass 1 clears the weights first
  int n_ctas;
};

// A sequence as the call sees it: tiles that hold a token some query sees (the first `ua`, then those from `ub0`).
struct ObSeq {
  int n, last;
  int ua, ub0, u;
  bool bad;
};
__device__ __forceinline__ ObSeq ob_seq(const ObserveParams& p, int b) {
  ObSeq s;
  const int raw = p.g.seq_lens[b];
  s.bad = raw < 0 || raw > p.g.max_seq_len;
  s.n = min(max(raw, 0), p.g.max_seq_len);
  s.last = min(max(p.rule.q_pos ? p.rule.q_pos[b] : s.n - 1, -1), kObNoToken - 1);
  s.ua = (s.n + kObTile - 1) / kObTile;
  s.ub0 = s.u = s.ua;
  if (p.positions == nullptr) {
    const View first = view_at(p.rule, b, max(s.last - p.n_obs + 1, -1));  // the query that looks back furthest
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

template <int DT, int PASS>
__global__ void __launch_bounds__(kObThreads, 1)
layer_observe_kernel(const __grid_constant__ ObserveParams p, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_q) {
  grid_dep_launch();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  // barriers: K full / empty per stage, Q full / empty per buffer, accumulator full / empty per group
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kObSmem);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kObMaxStages + 4 + 4);
  volatile int* s_abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* row_s = reinterpret_cast<float*>(tmem_slot + 2);     // [2 groups][256][2]: pass 1 (m, l) of the lanes; pass 2 lse, slope
  int* pos_s = reinterpret_cast<int*>(row_s + 2 * kObMaxRows * 2);  // [2 groups][128]
  int* pre_s = pos_s + 2 * kObTile;                           // [batch + 1]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = p.g.n_kv_heads, ps = p.g.page_size, shift = p.g.page_shift;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kObMaxStages, qfull0 = empty0 + 8 * kObMaxStages, qempty0 = qfull0 + 16;
  const uint32_t tfull0 = qempty0 + 16, tempty0 = tfull0 + 16;
  const int q_bytes = p.nt * kObTileBytes, q_half = p.nt * kObHalf;
  const uint32_t sq0 = smem_u32(smem), sk0 = sq0 + kObQBufs * q_bytes;
  const uint32_t tmem_cols = 2u * kObTile * p.nt;

  int bad = 0;
  for (int b = tid; b < p.g.batch; b += kObThreads) {
    const ObSeq s = ob_seq(p, b);
    bad |= s.bad ? 1 : 0;
    pre_s[b + 1] = s.u * H;
  }
  if (tid == 0) {
    for (int s = 0; s < kObMaxStages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(qfull0 + 8 * s, 1);
      mbar_init(qempty0 + 8 * s, 1);
      mbar_init(tfull0 + 8 * s, 1);
      mbar_init(tempty0 + 8 * s, 4);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), tmem_cols);
  tc_fence_before();
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
  tc_fence_after();
  const uint32_t tmem_d = *tmem_slot;
  const long long U = pre_s[p.g.batch];
  const int T = (int)min((long long)p.n_ctas, max(U, 1LL));  // no live CTA's share is empty
  const int cta = blockIdx.x;
  int x_begin = 0, n_x = 0;
  if (cta < T) {
    x_begin = (int)(U * cta / T);
    n_x = (int)(U * (cta + 1) / T) - x_begin;
  }
  constexpr int DIR = PASS == 1 ? 1 : -1;
  const int x_first = PASS == 1 ? x_begin : x_begin + n_x - 1;
  grid_dep_wait();
  if (bad) atomicOr(p.status, MC_FLAG_BAD_METADATA);

  if (PASS == 1 && p.zero) {  // tokens that no query sees keep no weight: all are cleared, pass 2 adds
    for (int s = cta; s < p.g.batch * H; s += gridDim.x) {
      const int b = s / H, g = s - b * H;
      const int n = min(max(p.g.seq_lens[b], 0), p.g.max_seq_len);
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
    // ===================== producer =====================
    ObCursor c;
    if (n_x > 0) c.seek(pre_s, p.g.batch, H, x_first);
    bool first = true, ok = true;
    int seg = 0;
    ObSeq sq = {};
    int sq_b = -1;
    bool has = false;  // this lane has a page of the tile
    // page id of this lane's page of the current tile, one tile ahead (a tile has at most 8 pages)
    auto tile_page = [&](const ObCursor& d) {
      if (d.b != sq_b) {
        sq = ob_seq(p, d.b);
        sq_b = d.b;
      }
      const int t = (d.k < sq.ua ? d.k : sq.ub0 + d.k - sq.ua) * kObTile + (lane << shift);
      has = lane < (kObTile >> shift) && t < sq.n;
      return has ? p.g.block_table[(size_t)d.b * p.g.max_pages_per_seq + (t >> shift)] : 0;
    };
    int page = n_x > 0 ? tile_page(c) : 0;
    for (int i = 0; i < n_x && ok; ++i) {
      if (first) {
        const int qb = seg & 1;
        if (seg >= 2) ok = __all_sync(0xffffffffu, mbar_wait(qempty0 + 8 * qb, ((seg >> 1) - 1) & 1, s_abort, p.status));
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
      }
      const int s = i % p.stages;
      if (i >= p.stages) ok = __all_sync(0xffffffffu, mbar_wait(empty0 + 8 * s, ((i / p.stages) - 1) & 1, s_abort, p.status));
      if (!ok) break;
      const int here = page;
      const bool copies = has;
      const ObCursor now = c;
      first = last_of_seg(c, i);
      if (first) ++seg;
      if (i + 1 < n_x) {
        advance(c, x_first + DIR * (i + 1));
        page = tile_page(c);
      }
      const uint32_t bar = full0 + 8 * s, dst = sk0 + s * kObTileBytes;
      const int n_copy = __popc(__ballot_sync(0xffffffffu, copies));
      if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n_copy * 2 * ps * 128));
      __syncwarp();
      if (copies) {
        int pg = here;
        if (!page_ok(p.g, pg)) {  // never an address: page 0 is read in its place and the call flagged
          atomicOr(p.status, MC_FLAG_BAD_METADATA);
          pg = 0;
        }
        const int y = (pg * H + now.g) * ps;
        tma_load_2d(dst + lane * ps * 128, &map_k, 0, y, bar);
        tma_load_2d(dst + kObHalf + lane * ps * 128, &map_k, 64, y, bar);
      }
      __syncwarp();
    }
  } else if (warp == 1) {
    // ===================== tensor-core issue =====================
    if (lane == 0) {
      ObCursor c;
      if (n_x > 0) c.seek(pre_s, p.g.batch, H, x_first);
      int seg = 0;
      bool first = true;
      const int n_cols = PASS == 1 ? kObTile : (p.rows + 15) / 16 * 16;
      const uint32_t idesc = umma_idesc<DT, 8>() - (1u << 17) + ((uint32_t)(n_cols >> 3) << 17);
      for (int i = 0; i < n_x; ++i) {
        const int s = i % p.stages, buf = i & 1, qb = seg & 1;
        if (first && !mbar_wait(qfull0 + 8 * qb, (seg >> 1) & 1, s_abort, p.status)) break;
        if (i >= 2 && !mbar_wait(tempty0 + 8 * buf, ((i >> 1) - 1) & 1, s_abort, p.status)) break;
        if (!mbar_wait(full0 + 8 * s, (i / p.stages) & 1, s_abort, p.status)) break;
        tc_fence_after();
        const uint32_t d = tmem_d + buf * kObTile * p.nt;
        const uint32_t qa = sq0 + qb * q_bytes, ka = sk0 + s * kObTileBytes;
        for (int tt = 0; tt < (PASS == 1 ? p.nt : 1); ++tt) {
#pragma unroll
          for (int k = 0; k < kHeadDim / 16; ++k) {
            const uint64_t dq = smem_desc_k128(qa + (k >> 2) * q_half + tt * kObHalf) + (uint64_t)(2 * (k & 3));
            const uint64_t dk = smem_desc_k128(ka + (k >> 2) * kObHalf) + (uint64_t)(2 * (k & 3));
            if (PASS == 1) umma_f16(d + tt * kObTile, dq, dk, idesc, k > 0 ? 1u : 0u);
            else umma_f16(d, dk, dq, idesc, k > 0 ? 1u : 0u);
          }
        }
        umma_commit(empty0 + 8 * s);
        first = last_of_seg(c, i);
        if (first) {
          umma_commit(qempty0 + 8 * qb);
          ++seg;
        }
        umma_commit(tfull0 + 8 * buf);
        if (i + 1 < n_x) advance(c, x_first + DIR * (i + 1));
      }
    }
  } else {
    // ===================== scores =====================
    const int grp = (warp - 2) >> 2, quad = warp & 3, gl = quad * 32 + lane;  // gl: this thread's tensor-memory lane
    const uint32_t tbuf = tmem_d + grp * kObTile * p.nt + ((uint32_t)(quad * 32) << 16);
    float* row_g = row_s + grp * kObMaxRows * 2;
    int* pos_g = pos_s + grp * kObTile;
    const bool no_max = p.rule.cap_log2 > 0.f && p.rule.cap_log2 <= 100.f && p.rule.slopes == nullptr;
    ObCursor c;
    if (n_x > 0) c.seek(pre_s, p.g.batch, H, x_first);
    bool first = true;
    ObSeq sq = {};
    float m[2], l[2], slope[2];  // pass 1: this lane's row of each row tile
    View vw[2];
    bool live[2];
    const int copy = gl / p.rp, c_lo = copy * (kObTile / p.rep), c_n = kObTile / p.rep;  // pass 1: this copy's columns
    for (int i = 0; i < n_x; ++i) {  // (also after a wait that ran out: the group's barriers stay matched)
      if (first) {
        sq = ob_seq(p, c.b);
        if (PASS == 1) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            const int r = tt * kObTile + gl % p.rp;
            m[tt] = no_max ? 0.f : -INFINITY;
            l[tt] = 0.f;
            live[tt] = tt < p.nt && copy < p.rep && r < p.rows;
            vw[tt] = view_at(p.rule, c.b, max(sq.last - p.n_obs + 1 + (live[tt] ? r / p.nq : 0), -1));
            slope[tt] = live[tt] && p.rule.slopes ? p.rule.slopes[c.g * p.nq + r % p.nq] * kLog2e : 0.f;
          }
        } else {
          // log-sum-exp of every row, from the partial sums of the CTAs that share the segment
          const long long x0 = pre_s[c.b] + (long long)c.g * c.u;
          const int c0 = (int)(((x0 + 1) * T - 1) / U), c1 = (int)(((x0 + c.u) * T - 1) / U);
          group_sync(grp);  // everybody has done with the segment before
          for (int r = gl; r < p.rows; r += kObTile) {
            float mm = -INFINITY, ll = 0.f;
            for (int cc = c0; cc <= c1; ++cc) {
              const float4 v = *reinterpret_cast<const float4*>(p.part_ml + ((size_t)(cc + c.b * H + c.g) * p.rows + r) * 4);
              const float M = fmaxf(mm, fmaxf(v.x, v.z));
              ll = (ll == 0.f ? 0.f : ll * exp2f(mm - M)) + (v.y == 0.f ? 0.f : v.y * exp2f(v.x - M)) +
                   (v.w == 0.f ? 0.f : v.w * exp2f(v.z - M));
              mm = M;
            }
            row_g[r] = ll == 0.f ? INFINITY : mm + log2f(ll);  // (a row that saw nothing gives nothing)
            row_g[kObMaxRows + r] = p.rule.slopes ? p.rule.slopes[c.g * p.nq + r % p.nq] * kLog2e : 0.f;
          }
          group_sync(grp);
        }
      }
      first = last_of_seg(c, i);
      if ((i & 1) == grp) {
        const int t0 = (c.k < sq.ua ? c.k : sq.ub0 + c.k - sq.ua) * kObTile;
        // a tile that every query sees whole needs no masks
        const int qp0 = max(sq.last - p.n_obs + 1, -1);
        const View v0 = view_at(p.rule, c.b, qp0), v1 = view_at(p.rule, c.b, sq.last);
        const bool whole = p.positions == nullptr && t0 + kObTile <= sq.n && t0 + kObTile - 1 <= qp0 &&
                           (t0 + kObTile <= v0.prefix || t0 >= v1.lo_pos);
        const bool easy = whole && p.rule.slopes == nullptr;
        // this thread's token: position, and in pass 2 where its weight goes
        const int t = t0 + gl;
        int pos = t < sq.n ? t : kObNoToken;
        float* dst = nullptr;
        if (t < sq.n && (PASS == 2 || p.positions)) {
          const int page = p.g.block_table[(size_t)c.b * p.g.max_pages_per_seq + (t >> shift)];
          const size_t at = ((size_t)page * H + c.g) * ps + (t & (ps - 1));
          if (page_ok(p.g, page)) {
            dst = p.weights + at;
            if (p.positions) pos = p.positions[at];
          }
        }
        if (PASS == 1 && !easy) {
          group_sync(grp);
          pos_g[gl] = pos;
          group_sync(grp);
        }
        float w_old = 0.f;
        if (PASS == 2 && p.add && dst) w_old = *dst;
        const bool good = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * grp, (i >> 1) & 1, s_abort, p.status));
        tc_fence_after();
        if (!good) {
        } else if (PASS == 1) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            if (tt * kObTile + (quad * 32) % p.rp >= p.rows) continue;  // (no lane of this warp has a row)
            float mr = m[tt], lr = l[tt];
            for (int c0 = 0; c0 < c_n; c0 += 32) {
              uint32_t raw[32];
              tmem_ld32(tbuf + tt * kObTile + c_lo + c0, raw);
              float s[32];
#pragma unroll
              for (int k = 0; k < 32; ++k) s[k] = score_of(p.rule, __uint_as_float(raw[k]));
              if (!easy) {
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                  const int pk = pos_g[c_lo + c0 + k];
                  s[k] = vw[tt].sees(pk) ? fmaf(-slope[tt], (float)(vw[tt].q_pos - pk), s[k]) : -INFINITY;
                }
              }
              if (!no_max) {
                float mx = s[0];
#pragma unroll
                for (int k = 1; k < 32; ++k) mx = fmaxf(mx, s[k]);
                if (mx > mr) {
                  lr *= exp2f(mr - mx);  // (l = 0 while m = -inf)
                  mr = mx;
                }
              }
              const float mb = mr == -INFINITY ? 0.f : mr;
              float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                sum0 += exp2f(s[k] - mb);
                sum1 += exp2f(s[k + 1] - mb);
              }
              lr += sum0 + sum1;
            }
            m[tt] = mr;
            l[tt] = lr;
          }
        } else {
          float w0 = 0.f, w1 = 0.f;
          for (int r0 = 0; r0 < p.rows; r0 += 32) {
            uint32_t raw[32];
            tmem_ld32(tbuf + r0, raw);
            const int nr = min(32, p.rows - r0);
            if (easy && nr == 32) {
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                w0 += exp2f(score_of(p.rule, __uint_as_float(raw[k])) - row_g[r0 + k]);
                w1 += exp2f(score_of(p.rule, __uint_as_float(raw[k + 1])) - row_g[r0 + k + 1]);
              }
            } else {
#pragma unroll
              for (int k = 0; k < 32; ++k) {
                if (k < nr) {
                  const int r = r0 + k;
                  float s = score_of(p.rule, __uint_as_float(raw[k]));
                  bool sees = true;
                  if (!easy) {
                    const int qp = max(qp0, sq.last - p.n_obs + 1 + r / p.nq);
                    const int lo = p.rule.window > 0 ? max(p.rule.doc_start ? p.rule.doc_start[c.b] : 0, qp - p.rule.window + 1) : v0.lo_pos;
                    sees = pos <= qp && (pos < v0.prefix || pos >= lo);
                    s = fmaf(-row_g[kObMaxRows + r], (float)(qp - pos), s);
                  }
                  if (sees) w0 += exp2f(s - row_g[r]);
                }
              }
            }
          }
          if (dst) *dst = w_old + (w0 + w1);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty0 + 8 * grp);
      }
      if (PASS == 1 && first) {
        // the copies of a row meet; one partial result per (CTA, segment, group)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          if (tt >= p.nt) continue;
          group_sync(grp);
          row_g[2 * gl] = l[tt] == 0.f ? -INFINITY : m[tt];
          row_g[2 * gl + 1] = live[tt] ? l[tt] : 0.f;
          group_sync(grp);
          const int r = tt * kObTile + gl;
          if (gl < p.rp && r < p.rows) {
            float mm = -INFINITY, ll = 0.f;
            for (int k = 0; k < p.rep; ++k) {
              const float mk = row_g[2 * (k * p.rp + gl)], lk = row_g[2 * (k * p.rp + gl) + 1];
              const float M = fmaxf(mm, mk);
              ll = (ll == 0.f ? 0.f : ll * exp2f(mm - M)) + (lk == 0.f ? 0.f : lk * exp2f(mk - M));
              mm = M;
            }
            float* o = p.part_ml + (((size_t)(cta + c.b * H + c.g) * p.rows + r) * 2 + grp) * 2;
            o[0] = mm;
            o[1] = ll;
          }
        }
      }
      if (i + 1 < n_x) advance(c, x_first + DIR * (i + 1));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*s_abort) {  // let copies in flight land before the CTA's memory is released
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
  if (warp == 1) tmem_dealloc(tmem_d, tmem_cols);
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kObMaxCtas = 256;
size_t layer_observe_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int n_obs) {
  const size_t rows = (size_t)n_obs * (cfg->n_q_heads / cfg->n_kv_heads);
  return align_up(((size_t)kObMaxCtas + (size_t)bt->batch * cfg->n_kv_heads) * rows * 4 * sizeof(float), 256);
}

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
  op.n_q_heads = cfg->n_q_heads;
  op.rows = n_obs * op.nq;
  op.nt = op.rows > kObTile ? 2 : 1;
  op.rp = op.rows > 64 ? 128 : (op.rows > 32 ? 64 : 32);
  op.rep = kObTile / op.rp;
  op.jt = std::min(n_obs, kObTile / op.nq);
  op.stages = op.nt == 1 ? kObMaxStages : 2;
  const bool hidden_tiles = opts->window > 0 || opts->doc_start != nullptr || opts->q_pos != nullptr;
  op.zero = !(flags & MC_LAYER_ACCUMULATE) && hidden_tiles;
  op.add = (flags & MC_LAYER_ACCUMULATE) || hidden_tiles;
  const long long max_tiles = (long long)bt->batch * cfg->n_kv_heads * ((bt->max_seq_len + kObTile - 1) / kObTile);
  op.n_ctas = (int)std::max<long long>(1, std::min<long long>(std::min(n_sm, kObMaxCtas), max_tiles));
  CUtensorMap map_k, map_q;
  const uint64_t rows = (uint64_t)bt->n_pages * cfg->n_kv_heads * cfg->page_size;
  if (mc_status st = make_map(&map_k, cfg->dtype, layer->k_pool, rows, kHeadDim, cfg->page_size)) return st;
  if (mc_status st = make_map3(&map_q, cfg->dtype, q, (uint64_t)bt->batch * n_obs, cfg->n_q_heads, kHeadDim, op.jt, op.nq)) return st;
  const size_t smem = 1024 + kObSmem + (2 * kObMaxStages + 8) * 8 + 8 + 2 * kObMaxRows * 2 * 4 + 2 * kObTile * 4 + (size_t)(bt->batch + 1) * 4;
  for (int pass = 1; pass <= 2; ++pass) {
    auto* kern = cfg->dtype == MC_F16 ? (pass == 1 ? layer_observe_kernel<MC_F16, 1> : layer_observe_kernel<MC_F16, 2>)
                                      : (pass == 1 ? layer_observe_kernel<MC_BF16, 1> : layer_observe_kernel<MC_BF16, 2>);
    MC_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    MC_CUDA_CHECK(launch_pdl(kern, dim3(op.n_ctas), dim3(kObThreads), smem, stream, op, map_k, map_q));
  }
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
