// Single-query decode attention over one layer held in 4 bits (keys per channel over a page of 32 tokens, values per token
// over 32 channels), the layers below MiniCache's start layer when the model's caches are 4-bit.
//
//   s_i   = sum_c (q_c scale_c) code_ic + sum_c q_c zero_c        (page by page: scale and zero belong to a page's channel)
//   out_c = sum_i (p_i scale_ig) code_ic + sum_i p_i zero_ig      (g: the channel's group of 32)
//
// The group parameters move to the operand with few rows: a page's 4096 codes of K and of V meet the tensor cores as they
// are, 128 products q scale and 128 products p scale are formed in their place.  A four-bit integer needs no conversion:
// masked out of a word, the bits 0..3 of a half-word are the binary16 number code * 2^-24 and the bits 4..7 code * 2^-20
// (subnormal numbers and the lowest binade share their unit), which the tensor cores multiply exactly; the powers of two
// are taken out of the fp32 sums.  Five logic operations per eight codes of K are all that is done to them, four of V: there a whole
// byte, low nibble + 16 high, and 16 high go to two rows of the accumulator, whose difference is taken once at the end.
//   q scale (22 bits) is carried as two binary16 numbers, its rounding and the rest, in neighbouring columns of the B operand
// that one kv head's few query heads leave idle (eight query heads: two passes), with a power of two that follows the page's scales,
// so scores are as exact as fp32 sums make them.
// p is kept below 2^e, p scale below 2^15, e chosen from the page's scales and lowered like a running maximum that rises.
//
// Work: the complete pages that are seen (or selected), split equally over teams of warps, a warp per kv head in each (neighbouring
// warps stream neighbouring tiles of a page).  A warp is a pipeline of its own with a ring of stages of one tile (5 KB: codes and
// parameters of K and V), two copied with the tensor map's swizzle so that ldmatrix and 16-byte loads meet no bank conflicts.
// A sequence's begun page and the step's new row, 16-bit rows, are a piece of their own: attended straight from global memory
// while the first tiles are on their way, and the new row appended.  Partial results are joined by a second kernel.
//
// Measured, from a CUDA graph: 8 x 4109 tokens of 32 heads 40.0 us (170 MB: 25.9 us at a copy's rate, 28.5 for a kernel that only reads
// them), 16 x 8192 of 8 kv heads under 32, capped, 43.8 us, under 64 without a cap 48.3 us.  Bound by how the work is started, streamed
// and joined more than by any unit: without arithmetic the 40.0 us are 33.0, without the combine kernel 36.8, without both 31.9 (copies
// of the kernel that leave these out), and no pipe is full (issue 51 %, ALU 45 %, tensor cores 19 %, memory 47 %).  A step in which
// every sequence's page fills: 74 us, as one warp quantises a page of K, then of V, from global memory.
#include <algorithm>

#include "mc_kernels.h"
#include "mc_layer.h"
#include "mc_layer_q4.cuh"
#include "mc_layer_q4.h"
#include "mc_mma.cuh"
#include "mc_pipe.cuh"
#include "mc_tc.cuh"

namespace mc {

// Twelve warps an SM fit 168 registers each (sixteen spill: 54 instead of 44 us); as two CTAs, so that the next kernel's first CTAs
// find room (one of twelve 43, two of six 40, three of four up to 64: starts packed unevenly).  Two stages: three 47, more requests
// outstanding than the memory serves well.
constexpr int kLqWarps = 6;
constexpr int kLqThreads = kLqWarps * 32;
constexpr int kLqCtasPerSm = 2;
constexpr int kLqStages = 2;
constexpr int kLqStageBytes = 2 * (kLqCodeBytes + kLqMetaBytes);
constexpr int kLqVCodes = kLqCodeBytes, kLqKMeta = 2 * kLqCodeBytes, kLqVMeta = kLqKMeta + kLqMetaBytes;  // within a stage
static_assert(kLqStageBytes % 1024 == 0, "the swizzle patterns repeat within 1 KB");

struct LayerQ4Params {
  Geom g;
  ScoreRule rule;
  const unsigned char* k_codes;
  const unsigned char* v_meta;
  unsigned char* pool[4];  // k_codes, k_meta, v_codes, v_meta (append)
  char* res_k;
  char* res_v;
  int32_t* status;
  const char* q;
  const char* k_new;
  const char* v_new;
  const int32_t* sel;     // selected pages or null
  const int32_t* counts;
  int sel_stride;
  float* part_o;   // [team + sequence][n_q_heads][128], then [sequence][n_q_heads][128] of the 16-bit rows
  float* part_ml;  // [...][2]
  int res_part;    // first row of the latter
  int4* pieces;    // [batch]: first team, number of teams that have pages of a sequence, whether it has 16-bit rows
  int nq, n_q_heads;
  int members, n_teams;  // warps of a team, teams
  int flags;
  unsigned short* out;
  float* lse;
};

// What every CTA keeps of a sequence.
struct Q4Seq : TokenView {
  bool append;  // (not where its length was out of range: the new row would land on cached ones)
};
// A sequence as the call sees it; `begun`: 1 if there are 16-bit rows (the begun page's, the step's new one).
__device__ __forceinline__ PageView q4_view(const LayerQ4Params& p, int b, int& begun, int& bad) {
  const int raw = __ldcg(p.g.seq_lens + b);
  bad |= (raw < 0 || raw > p.g.max_seq_len) ? 1 : 0;
  const int n = min(max(raw, 0), p.g.max_seq_len), n_tot = n + (p.k_new != nullptr ? 1 : 0);
  begun = n_tot > n / kLqPage * kLqPage ? 1 : 0;
  return page_view(p.rule, b, n, n_tot, n_tot - 1);
}
// Pages of sequence b, of n tokens, in the selection.
__device__ __forceinline__ int q4_selected(const LayerQ4Params& p, int b, int n, int& bad) {
  const int c = __ldcg(p.counts + b), most = min(p.sel_stride, n / kLqPage);
  bad |= (c < 0 || c > most) ? 1 : 0;
  return min(max(c, 0), most);
}

// The units of a call: all pages, sequence by sequence, then the begun pages, which count for kLqBegunUnits each: one waits for the
// memory behind the stream and is not pipelined, 3.5 us against a page's 1.5.  (8 x 4109 tokens of 32 heads / 16 x 64 selected pages of
// 8: one unit 57 / 25 us, two 48 / 19, three 39.6 / 17.7, four 38.6 / 17.6, five 41 / 17.5; rows prefetched to L2 ahead: no gain.)
constexpr int kLqBegunUnits = 4;
struct Q4Prefix {
  int* pages;  // [batch + 1] exclusive prefixes
  int* begun;
};
__device__ __forceinline__ Q4Prefix q4_prefix_at(void* smem, int batch) {
  Q4Prefix f;
  f.pages = reinterpret_cast<int*>(smem);
  f.begun = f.pages + batch + 1;
  return f;
}
__device__ __forceinline__ void q4_scan(const Q4Prefix& f, int batch) {
  __syncthreads();
  if (threadIdx.x < 64) scan_warp(threadIdx.x < 32 ? f.pages : f.begun, batch);
  __syncthreads();
}
__device__ __forceinline__ int q4_total(const Q4Prefix& f, int batch) { return f.pages[batch] + kLqBegunUnits * f.begun[batch]; }
__device__ __forceinline__ int q4_live_teams(const LayerQ4Params& p, int units) { return min(p.n_teams, max(units, 1)); }

// A warp's share: of the pages [x0, x1) and the begun pages [g0, g1) of the batch the kv heads member, member + members, ...
struct Q4Share {
  int team, member, n_heads;
  int x0, x1, g0, g1;
};
__device__ __forceinline__ Q4Share q4_share(const LayerQ4Params& p, const Q4Prefix& f, int warp) {
  Q4Share s;
  s.team = warp / p.members;
  s.member = warp - s.team * p.members;
  s.n_heads = (p.g.n_kv_heads - s.member + p.members - 1) / p.members;
  const int pages = f.pages[p.g.batch], units = q4_total(f, p.g.batch), teams = q4_live_teams(p, units);
  int u0 = 0, u1 = 0;
  if (s.team < teams) {
    u0 = (int)((long long)units * s.team / teams);
    u1 = (int)((long long)units * (s.team + 1) / teams);
  }
  s.x0 = min(u0, pages);
  s.x1 = min(u1, pages);
  s.g0 = (max(u0 - pages, 0) + kLqBegunUnits - 1) / kLqBegunUnits;  // (a begun page is its first unit's owner's)
  s.g1 = (max(u1 - pages, 0) + kLqBegunUnits - 1) / kLqBegunUnits;
  return s;
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c) {
  const __half2 r = __hfma2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b), *reinterpret_cast<__half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t h2_max(uint32_t a, uint32_t b) {
  const __half2 r = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// D = A B (mma_rows without an addend: no registers to be cleared)
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// c + (low or high half of a) (high half of b), in binary32: sm_100's mixed-precision FMA (a tensor-core row of zeros costs
// eight of its cycles and the halves' rearrangement besides).
__device__ __forceinline__ float fma_lo_hi(uint32_t a, uint32_t b, float c) {
  float r;
  asm("{\n\t.reg .b16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %1;\n\tmov.b32 {bl, bh}, %2;\n\tfma.rn.f32.f16 %0, al, bh, %3;\n\t}"
      : "=f"(r)
      : "r"(a), "r"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float fma_hi_hi(uint32_t a, uint32_t b, float c) {
  float r;
  asm("{\n\t.reg .b16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %1;\n\tmov.b32 {bl, bh}, %2;\n\tfma.rn.f32.f16 %0, ah, bh, %3;\n\t}"
      : "=f"(r)
      : "r"(a), "r"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t lows(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t highs(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

// The 16-bit rows of one (sequence, kv head), by a warp: the begun page's and the step's new one, up to 32 tokens, straight
// from global memory.  The k axis of the first product is the channels in the order in which a lane's 16-byte loads bring
// them; in the second a lane's rows and channels are the ones the codes' kernel uses, so that outputs leave alike.
template <int DT>
__device__ __noinline__ void q4_begun_page(const LayerQ4Params& p, const Q4Seq v, int b, int head) {
  const int lane = threadIdx.x & 31, row = lane >> 2, t4 = lane & 3, colp = 2 * t4;
  const int nq = p.nq, H = p.g.n_kv_heads;
  const int n = v.n, base = n / kLqPage * kLqPage, n_tot = n + (p.k_new != nullptr ? 1 : 0);
  const size_t at = ((size_t)b * H + head) * kLqResBytes, new_at = ((size_t)b * H + head) * kRowBytes;
  const size_t prow = (size_t)p.res_part + (size_t)b * p.n_q_heads + head * nq;
  uint32_t seen = 0;  // bit r: token base + r is attended
  {
    const int t = base + lane;
    seen = __ballot_sync(0xffffffffu, t < n_tot && v.sees(t));
  }
  float acc[8][4];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[j][k] = 0.f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  if (seen != 0) {
    auto row_ptr = [&](bool keys, int r) {
      return base + r == n ? (keys ? p.k_new : p.v_new) + new_at : (keys ? p.res_k : p.res_v) + at + (size_t)r * kRowBytes;
    };
    uint4 qf[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      qf[j] = make_uint4(0u, 0u, 0u, 0u);
      if (row < nq) qf[j] = *reinterpret_cast<const uint4*>(p.q + ((size_t)b * p.n_q_heads + head * nq + row) * kRowBytes + 64 * t4 + 16 * j);
    }
    float sc[2][4];
    uint2 vr[2][4][4];  // [16 tokens][token 2 t4, + 1, + 8, + 9][channel group]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool any = ((seen >> (16 * h)) & 0xffffu) != 0;
      uint4 ka[2][4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * h + 8 * e + row;
        const char* src = row_ptr(true, r) + 64 * t4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ka[e][j] = make_uint4(0u, 0u, 0u, 0u);
          if (any && ((seen >> r) & 1u)) ka[e][j] = *reinterpret_cast<const uint4*>(src + 16 * j);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 16 * h + (e >> 1) * 8 + colp + (e & 1);
        const char* src = row_ptr(false, r) + 8 * row;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          vr[h][e][g] = make_uint2(0u, 0u);
          if (any && ((seen >> r) & 1u)) vr[h][e][g] = *reinterpret_cast<const uint2*>(src + 64 * g);
        }
      }
      float d[2][4] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mma_rows<DT>(d[0], ka[0][j].x, ka[1][j].x, ka[0][j].y, ka[1][j].y, qf[j].x, qf[j].y);
        mma_rows<DT>(d[1], ka[0][j].z, ka[1][j].z, ka[0][j].w, ka[1][j].w, qf[j].z, qf[j].w);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) sc[h][k] = d[0][k] + d[1][k];
      const int p0 = base + 16 * h + row, p8 = p0 + 8;
      const bool v0 = (seen >> (16 * h + row)) & 1u, v8 = (seen >> (16 * h + row + 8)) & 1u;
      scores_of(p.rule, sc[h]);  // (what is not seen came as zeros)
      if (p.rule.slopes) {
        const float e0 = (float)(v.q_pos - p0), e8 = (float)(v.q_pos - p8);
        const float sl0 = colp < nq ? p.rule.slopes[head * nq + colp] * kLog2e : 0.f;
        const float sl1 = colp + 1 < nq ? p.rule.slopes[head * nq + colp + 1] * kLog2e : 0.f;
        sc[h][0] = fmaf(-sl0, e0, sc[h][0]);
        sc[h][1] = fmaf(-sl1, e0, sc[h][1]);
        sc[h][2] = fmaf(-sl0, e8, sc[h][2]);
        sc[h][3] = fmaf(-sl1, e8, sc[h][3]);
      }
      if (!v0) sc[h][0] = sc[h][1] = -INFINITY;
      if (!v8) sc[h][2] = sc[h][3] = -INFINITY;
      m0 = fmaxf(m0, fmaxf(sc[h][0], sc[h][2]));
      m1 = fmaxf(m1, fmaxf(sc[h][1], sc[h][3]));
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, o));
      m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, o));
    }
    const float b0 = m0 == -INFINITY ? 0.f : m0, b1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float e0 = ex2(sc[h][0] - b0), e1 = ex2(sc[h][1] - b1), e2 = ex2(sc[h][2] - b0), e3 = ex2(sc[h][3] - b1);
      l0 += e0 + e2;
      l1 += e1 + e3;
      const uint32_t pb0 = transpose_8x8(Elem<DT>::pack(e0, e1)), pb1 = transpose_8x8(Elem<DT>::pack(e2, e3));
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        mma_rows<DT>(acc[2 * g], lows(vr[h][0][g].x, vr[h][1][g].x), highs(vr[h][0][g].x, vr[h][1][g].x), lows(vr[h][2][g].x, vr[h][3][g].x),
                     highs(vr[h][2][g].x, vr[h][3][g].x), pb0, pb1);
        mma_rows<DT>(acc[2 * g + 1], lows(vr[h][0][g].y, vr[h][1][g].y), highs(vr[h][0][g].y, vr[h][1][g].y),
                     lows(vr[h][2][g].y, vr[h][3][g].y), highs(vr[h][2][g].y, vr[h][3][g].y), pb0, pb1);
      }
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, o);
      l1 += __shfl_xor_sync(0xffffffffu, l1, o);
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = colp + e;
    if (r >= nq) continue;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(p.part_o + (prow + r) * kHeadDim + 32 * g + 4 * row) =
          make_float4(acc[2 * g][e], acc[2 * g][2 + e], acc[2 * g + 1][e], acc[2 * g + 1][2 + e]);
    if (row == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * (prow + r)) = make_float2(e ? m1 : m0, e ? l1 : l0);
  }
  if (v.append) {
    const int slot = n & (kLqPage - 1);
    const int ch = lane & 15;  // lanes 0 .. 15: the new K row's chunks, 16 .. 31: the V row's
    *reinterpret_cast<uint4*>((lane < 16 ? p.res_k : p.res_v) + at + slot * kRowBytes + 16 * ch) =
        *reinterpret_cast<const uint4*>((lane < 16 ? p.k_new : p.v_new) + new_at + 16 * ch);
    if (slot == kLqPage - 1) {  // the row completes a page
      __syncwarp();             // (which other lanes of the warp have just written)
      const int page = checked_page(p.g, b, n / kLqPage, p.status);
#pragma unroll 1
      for (int tensor = 0; tensor < 2 && page >= 0; ++tensor) {
        const char* src = (tensor == 0 ? p.res_k : p.res_v) + at + 16 * ch;
        const size_t tile = (size_t)page * H + head;
        lq_quantise<DT>(tensor == 0, [&](int t) { return *reinterpret_cast<const uint4*>(src + t * kRowBytes); },
                        p.pool[2 * tensor] + tile * kLqCodeBytes, p.pool[2 * tensor + 1] + tile * kLqMetaBytes);
      }
    }
  }
}

// q scale as two binary16 numbers loses what is below 2^-25.  A query's largest entry is brought to [2^kLqQueryExp, 2^(kLqQueryExp + 1)),
// and a page whose largest key scale is in [2^-kLqQueryExp, 2^(15 - kLqQueryExp)) is met as it is: products are below 2^16, and the
// largest that the page allows is 1 or more, so that 2^-25 of that one is what any of its products may lose.  Other pages (keys that
// spread over more than 480, or less than 0.015 in every channel) have a power of two taken out of their scales first.
constexpr int kLqQueryExp = 10;
constexpr uint32_t kLqLeastTop = (uint32_t)(15 - kLqQueryExp) << 10, kLqTops = (uint32_t)(30 - kLqQueryExp) << 10;  // (binary16, as integers)
static_assert(kLqQueryExp < 15, "normal numbers");

// Brings the largest of a page's key scales, `top` (binary16, as an integer), to [2^3, 2^4), where they lie; 2^24 over the factor.
__device__ __noinline__ float q4_rescale_keys(uint32_t k_meta, uint32_t top) {
  const int lane = threadIdx.x & 31;
  const int by = min(max(3 + 127 - (__float_as_int(half_lo(top)) >> 23), -12), 27);  // (a subnormal scale is a normal binary32 number)
  const float f = __int_as_float((127 + by) << 23);
  const uint4 u = lds16(k_meta + 16 * lane);
  uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int c = 0; c < 4; ++c) w[c] = (w[c] & 0xffff0000u) | (uint32_t)__half_as_ushort(__float2half_rn(half_lo(w[c]) * f));
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(k_meta + 16 * lane), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (ahead of the copy that follows into this place)
  __syncwarp();
  return __int_as_float((127 + 24 - by) << 23);
}

// WIDE: eight query heads per kv head, a column of B each; else up to four, two columns each.
template <int DT, bool WIDE>
__global__ void __launch_bounds__(kLqThreads, kLqCtasPerSm)
layer_q4_split_kernel(const __grid_constant__ LayerQ4Params p, const __grid_constant__ CUtensorMap map_km,
                      const __grid_constant__ CUtensorMap map_vc) {
  grid_dep_launch();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kLqWarps * kLqStages * kLqStageBytes);
  Q4Seq* seq_s = reinterpret_cast<Q4Seq*>(bars + kLqWarps * kLqStages);
  Q4Prefix pre = q4_prefix_at(seq_s + p.g.batch, p.g.batch);
  volatile int* s_abort = pre.begun + p.g.batch + 1;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = lane >> 2, t4 = lane & 3;
  const int H = p.g.n_kv_heads, nq = p.nq;

  if (tid == 32) {
    prefetch_map(&map_km);
    prefetch_map(&map_vc);
  }
  if (tid == 0) {
    for (int s = 0; s < kLqWarps * kLqStages; ++s) mbar_init(smem_u32(bars + s), 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // (lengths, block table and score options are the caller's: read before the wait; a selection is what the kernel ahead wrote)
  if (tid * 32 < (long long)p.g.batch * p.g.max_pages_per_seq)  // the block table, or its first lines, on its way to L2 meanwhile
    asm volatile("prefetch.global.L2 [%0];" ::"l"(p.g.block_table + tid * 32));
  int bad = 0;
  for (int b = tid; b < p.g.batch; b += kLqThreads) {
    int begun;
    int no_len = 0;
    const PageView v = q4_view(p, b, begun, no_len);
    bad |= no_len;
    pre.pages[b + 1] = v.u;
    pre.begun[b + 1] = begun;
    Q4Seq s;
    static_cast<TokenView&>(s) = v;
    s.append = (p.flags & MC_LAYER_APPEND) != 0 && no_len == 0;
    seq_s[b] = s;
  }
  if (p.sel != nullptr) {
    grid_dep_wait();
    for (int b = tid; b < p.g.batch; b += kLqThreads) pre.pages[b + 1] = q4_selected(p, b, seq_s[b].n, bad);
  }
  q4_scan(pre, p.g.batch);

  const Q4Share sh = q4_share(p, pre, blockIdx.x * kLqWarps + warp);
  const int nx = sh.x1 - sh.x0;
  const int n_tiles = nx * sh.n_heads;  // of this warp: head by head, page by page

  struct Tile {
    int page;  // raw page id
    int meta;  // kv head, or -1 where nothing is to be looked up
  };
  auto load_tile = [&](int i) {
    Tile t;
    t.page = 0;
    t.meta = -1;
    if (i >= n_tiles) return t;
    const int hd = sh.n_heads == 1 ? 0 : i / nx, x = sh.x0 + i - hd * nx;
    const int b = seq_of_item(pre.pages, p.g.batch, x), k = x - pre.pages[b];
    t.meta = sh.member + hd * p.members;
    int slot;
    if (p.sel == nullptr) {
      const int ua = seq_s[b].head_pages();
      slot = k < ua ? k : seq_s[b].tail_page(ua) + k - ua;
    } else {
      slot = __ldcg(p.sel + ((size_t)b * H + t.meta) * p.sel_stride + k);
      if ((unsigned)slot >= (unsigned)seq_s[b].full()) slot = -1;  // (flagged when its turn comes)
    }
    if (slot >= 0) t.page = slot < p.g.max_pages_per_seq ? p.g.block_table[(size_t)b * p.g.max_pages_per_seq + slot] : -1;
    return t;
  };
  // the pools' tile; a page id outside the pools reads page 0 and is flagged
  auto tile_of = [&](const Tile& t) {
    if (t.meta < 0) return 0;
    int page = t.page;
    if (!page_ok(p.g, page)) {
      atomicOr(p.status, MC_FLAG_BAD_METADATA);
      page = 0;
    }
    return page * H + t.meta;
  };
  const Tile first = load_tile(lane);
  if (p.sel == nullptr) grid_dep_wait();
  if (bad && blockIdx.x == 0) atomicOr(p.status, MC_FLAG_BAD_METADATA);  // (every thread has looked at other sequences)
  if (blockIdx.x == gridDim.x - 1) {  // for the kernel behind
    const long long units = q4_total(pre, p.g.batch);
    const int teams = q4_live_teams(p, (int)units);
    for (int b = tid; b < p.g.batch; b += kLqThreads) {
      const int u0 = pre.pages[b], u = pre.pages[b + 1] - u0;
      // the team of unit x is the last c with floor(units c / teams) <= x
      const int c0 = u > 0 ? (int)(((long long)(u0 + 1) * teams - 1) / units) : 0;
      const int c1 = u > 0 ? (int)(((long long)(u0 + u) * teams - 1) / units) : -1;
      p.pieces[b] = make_int4(c0, c1 - c0 + 1, pre.begun[b + 1] - pre.begun[b], 0);
    }
  }

  const uint32_t bar0 = smem_u32(bars + warp * kLqStages);
  const uint32_t st0 = smem_u32(smem) + warp * kLqStages * kLqStageBytes;
  // Copies run kLqStages - 1 tiles ahead: tile j into stage j % kLqStages.  `tiles`: a lane per tile, 32 of them.
  int tiles = tile_of(first);
  Tile ahead;
  int j = 0;
  auto issue = [&](uint32_t st_j, uint32_t bar_j) {
    if (j >= n_tiles) return;
    if ((j & 31) == 0 && j > 0) {
      tiles = tile_of(ahead);
      ahead = load_tile(j + 32 + lane);
    }
    const int y = __shfl_sync(0xffffffffu, tiles, j & 31);
    if (lane == 0) {
      mbar_expect_tx(bar_j, (uint32_t)kLqStageBytes);
      bulk_load(st_j, p.k_codes + (size_t)y * kLqCodeBytes, kLqCodeBytes, bar_j);
      tma_load_2d(st_j + kLqKMeta, &map_km, 0, y * 4, bar_j);
      tma_load_2d(st_j + kLqVCodes, &map_vc, 0, y * kLqPage, bar_j);
      bulk_load(st_j + kLqVMeta, p.v_meta + (size_t)y * kLqMetaBytes, kLqMetaBytes, bar_j);
    }
    ++j;
  };
  for (int i = 0; i < kLqStages - 1; ++i) issue(st0 + i * kLqStageBytes, bar0 + 8 * i);
  ahead = load_tile(32 + lane);
  for (int k = sh.g0; k < sh.g1; ++k) {  // the begun pages of the warp's share
    const int b = seq_of_item(pre.begun, p.g.batch, k);
    for (int hd = 0; hd < sh.n_heads; ++hd) q4_begun_page<DT>(p, seq_s[b], b, sh.member + hd * p.members);
  }

  uint32_t st_i = st0, bar_i = bar0, parity = 0;
  uint32_t st_free = st0 + (kLqStages - 1) * kLqStageBytes, bar_free = bar0 + 8 * (kLqStages - 1);  // the stage read last
  uint32_t km_off[4];  // where the lane's 16-byte chunks of the keys' parameters are: chunk c ^ t4 of row t4
#pragma unroll
  for (int c = 0; c < 4; ++c) km_off[c] = kLqKMeta + 128 * t4 + ((c ^ t4) << 4);
  const uint32_t k_off = row * 64 + 16 * t4;
  const uint32_t vc_off = kLqVCodes + (lane & 7) * 64 + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);
  const uint32_t vm_off = kLqVMeta + 32 * t4;

  for (int hd = 0; hd < sh.n_heads; ++hd) {
    const int head = sh.member + hd * p.members;
    for (int x = sh.x0; x < sh.x1;) {
      // ---- a piece: pages of one (sequence, kv head)
      const int b = seq_of_item(pre.pages, p.g.batch, x);
      const int k0 = x - pre.pages[b], k1 = min(sh.x1, pre.pages[b + 1]) - pre.pages[b];
      x += k1 - k0;
      const Q4Seq sq = seq_s[b];
      const int32_t* list = p.sel ? p.sel + ((size_t)b * H + head) * p.sel_stride : nullptr;
      const int ua = sq.head_pages(), ub0 = sq.tail_page(ua);
      int slot_next = list ? __ldcg(list + k0) : k0 < ua ? k0 : ub0 + k0 - ua;
      // the last page of the list that counted: the largest so far, which may lie in another warp's part (a lane's first entry comes
      // with the queries)
      int slot_last = list && lane < k0 ? __ldcg(list + lane) : -1;

      // Query pairs (channels 8w + i, 8w + i + 4 of the lane's 32), as binary16 with the row's power of two taken out: the
      // row's largest number becomes 2^10 to 2^11.  q_back, of the lane's result column(s), puts it back.
      uint32_t qh[16];
      float q_back, q_back1 = 0.f;
      {
        const int h = WIDE ? row : row >> 1;
        uint4 w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          w[c] = make_uint4(0u, 0u, 0u, 0u);
          if (h < nq) w[c] = *reinterpret_cast<const uint4*>(p.q + ((size_t)b * p.n_q_heads + head * nq + h) * kRowBytes + 64 * t4 + 16 * c);
        }
        float big = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t y[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = Elem<DT>::unpack(y[k]);
            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const int e = min(max(__float_as_int(big) >> 23, kLqQueryExp + 1), 253);
        const float f = __int_as_float((254 + kLqQueryExp - e) << 23);
        const float back = __int_as_float((e - kLqQueryExp) << 23);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t y[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
          uint32_t h2[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 v = Elem<DT>::unpack(y[k]);
            h2[k] = Elem<MC_F16>::pack(v.x * f, v.y * f);
          }
          qh[4 * c] = lows(h2[0], h2[2]);
          qh[4 * c + 1] = highs(h2[0], h2[2]);
          qh[4 * c + 2] = lows(h2[1], h2[3]);
          qh[4 * c + 3] = highs(h2[1], h2[3]);
        }
        // the lane's result columns are 2 t4 and 2 t4 + 1: rows 2 t4 and 2 t4 + 1 hold their queries
        q_back = __shfl_sync(0xffffffffu, back, 8 * t4);
        if (WIDE) q_back1 = __shfl_sync(0xffffffffu, back, 8 * t4 + 4);
      }
      if (list != nullptr) {
        if (slot_last >= sq.full()) slot_last = -1;
#pragma unroll 8
        for (int k = lane + 32; k < k0; k += 32) {
          const int e = __ldcg(list + k);
          if (e < sq.full()) slot_last = max(slot_last, e);
        }
        slot_last = __reduce_max_sync(0xffffffffu, max(slot_last, -1));
      }
      float sl0 = 0.f, sl1 = 0.f;
      if (p.rule.slopes) {
        const int h = WIDE ? 2 * t4 : t4;
        sl0 = h < nq ? p.rule.slopes[head * nq + h] * kLog2e : 0.f;
        if (WIDE) sl1 = p.rule.slopes[head * nq + h + 1] * kLog2e;
      }
      uint32_t qn[16];  // -q where the rounding is wanted, else 0 (a register each: a mask per product and page costs more)
#pragma unroll
      for (int c = 0; c < 16; ++c) qn[c] = WIDE || (row & 1) ? qh[c] ^ 0x80008000u : 0u;
      const bool unusual = p.rule.cap_log2 > 0.f || p.rule.slopes != nullptr;
      float acc[8][4], zacc[4];
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[c][k] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) zacc[k] = 0.f;
      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;  // of query head t4, or (WIDE) 2 t4 and 2 t4 + 1
      float ve = 0.f;          // probabilities are kept times 2^ve
      uint32_t scale_top = 0;  // the scale (binary16, as an integer) from which they no longer may be

      for (int k = k0; k < k1; ++k) {
        __syncwarp();  // (the stage of the tile before this one has been read)
        issue(st_free, bar_free);
        int slot = slot_next;
        if (list == nullptr) {
          slot_next = k + 1 == ua ? ub0 : slot + 1;
        } else {
          if (k + 1 < k1) slot_next = __ldcg(list + k + 1);
          const bool wrong = slot <= slot_last || slot < 0 || slot >= sq.full();
          if (wrong) {  // not above every one that counted, or no complete page: nothing of it is seen
            if (lane == 0) atomicOr(p.status, MC_FLAG_BAD_METADATA);
            slot = -1;
          } else {
            slot_last = slot;
          }
        }
        const int t0 = slot * kLqPage;
        const uint32_t sb = st_i;
        mbar_wait_lean(bar_i, parity, s_abort, p.status);  // (on a time-out the CTA only runs to its end)
        st_free = st_i;
        bar_free = bar_i;
        st_i += kLqStageBytes;
        bar_i += 8;
        if (st_i == st0 + kLqStages * kLqStageBytes) {
          st_i = st0;
          bar_i = bar0;
          parity ^= 1u;
        }
        // ---- scores of 32 tokens: two tiles of 16
        float dl[2][4], dh[2][4];  // low and high nibbles' sums
        float low = 0x1p24f, high;  // what takes the powers of two of the nibbles, and of the keys' scales, out of them
        float dz[4] = {};           // the zeros' sum of this lane's column and channels
        {
          uint4 c4[2][2];  // [tile][token row, row + 8]: 32 channels
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) c4[h][e] = lds16(sb + k_off + (16 * h + 8 * e) * 64);
          {  // (the latency of this, a load, a reduction and a branch, is 1.5 of 40 us; behind the products it costs 3 to 6)
            const uint4 u = lds16(sb + kLqKMeta + 16 * lane);
            const uint32_t top = __reduce_max_sync(0xffffffffu, h2_max(h2_max(u.x, u.y), h2_max(u.z, u.w)) & 0x7fffu);
            if (top - kLqLeastTop >= kLqTops - kLqLeastTop) low = q4_rescale_keys(sb + kLqKMeta, top);
          }
          high = low * 0x1p-4f;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint4 ma = lds16(sb + km_off[2 * (w & 1)] + 64 * (w >> 1)), mb = lds16(sb + km_off[2 * (w & 1) + 1] + 64 * (w >> 1));
            const uint32_t s4[4] = {lows(ma.x, mb.x), lows(ma.y, mb.y), lows(ma.z, mb.z), lows(ma.w, mb.w)};
            const uint32_t za[4] = {ma.x, ma.y, ma.z, ma.w}, zb[4] = {mb.x, mb.y, mb.z, mb.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              dz[c] = fma_lo_hi(qh[4 * w + c], za[c], dz[c]);
              dz[c] = fma_hi_hi(qh[4 * w + c], zb[c], dz[c]);
            }
            uint32_t bq[4], br[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t r = h2_mul(qn[4 * w + c], s4[c]);
              if (WIDE) {
                bq[c] = r ^ 0x80008000u;
                br[c] = h2_fma(qh[4 * w + c], s4[c], r);
              } else {
                bq[c] = h2_fma(qh[4 * w + c], s4[c], r);  // the product, or it less its rounding
              }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t c0 = w == 0 ? c4[h][0].x : w == 1 ? c4[h][0].y : w == 2 ? c4[h][0].z : c4[h][0].w;
              const uint32_t c8 = w == 0 ? c4[h][1].x : w == 1 ? c4[h][1].y : w == 2 ? c4[h][1].z : c4[h][1].w;
              const uint32_t u0 = c0 >> 8, u8 = c8 >> 8;
              const uint32_t a0 = c0 & 0x000f000fu, a1 = c8 & 0x000f000fu, a2 = u0 & 0x000f000fu, a3 = u8 & 0x000f000fu;
              const uint32_t h0 = c0 & 0x00f000f0u, h1 = c8 & 0x00f000f0u, h2 = u0 & 0x00f000f0u, h3 = u8 & 0x00f000f0u;
              if (w == 0) {
                mma_first(dl[h], a0, a1, a2, a3, bq[0], bq[2]);
                mma_first(dh[h], h0, h1, h2, h3, bq[1], bq[3]);
              } else {
                mma_rows<MC_F16>(dl[h], a0, a1, a2, a3, bq[0], bq[2]);
                mma_rows<MC_F16>(dh[h], h0, h1, h2, h3, bq[1], bq[3]);
              }
              if (WIDE) {
                mma_rows<MC_F16>(dl[h], a0, a1, a2, a3, br[0], br[2]);
                mma_rows<MC_F16>(dh[h], h0, h1, h2, h3, br[1], br[3]);
              }
            }
          }
        }
        // the zeros' sum over the lanes that share the column, then to the lanes that hold the column's results
        float z0 = (dz[0] + dz[1]) + (dz[2] + dz[3]), z1 = 0.f;
        z0 += __shfl_xor_sync(0xffffffffu, z0, 1);
        z0 += __shfl_xor_sync(0xffffffffu, z0, 2);
        if (WIDE) z1 = __shfl_sync(0xffffffffu, z0, 8 * t4 + 4);
        z0 = __shfl_sync(0xffffffffu, z0, 8 * t4);
        // tokens t0 + 16 h + row and + 8; not WIDE: sc[2 h + e] of query head t4; WIDE: sa of head 2 t4, sc of 2 t4 + 1
        float sc[4], sa[4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (WIDE) {
              sa[2 * h + e] = fmaf(dl[h][2 * e], low, fmaf(dh[h][2 * e], high, z0)) * q_back;
              sc[2 * h + e] = fmaf(dl[h][2 * e + 1], low, fmaf(dh[h][2 * e + 1], high, z1)) * q_back1;
            } else {
              sc[2 * h + e] = fmaf(dl[h][2 * e] + dl[h][2 * e + 1], low, fmaf(dh[h][2 * e] + dh[h][2 * e + 1], high, z0)) * q_back;
            }
          }
        // ---- masks, the scores' form, the distance bias
        if (!(p.rule.cap_log2 > 0.f)) {  // (behind q_back: their product may be no number where the score is one)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            sc[c] *= p.rule.scale_log2;
            if (WIDE) sa[c] *= p.rule.scale_log2;
          }
        }
        uint32_t hidden = 0;  // bit r: token t0 + r is not seen
        const bool whole = sq.all_of(t0) && slot >= 0;
        if (!whole || unusual) {
          if (!whole) {
            const int t = t0 + lane;
            hidden = ~__ballot_sync(0xffffffffu, slot >= 0 && sq.sees(t));
            if (p.rule.cap_log2 > 0.f) {  // (no say in which form of the cap the others take)
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if ((hidden >> (8 * c + row)) & 1u) sc[c] = sa[c] = 0.f;
            }
          }
          if (p.rule.cap_log2 > 0.f) {
            scores_of(p.rule, sc);
            if (WIDE) scores_of(p.rule, sa);
          }
          if (p.rule.slopes) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float dist = (float)(sq.q_pos - (t0 + 8 * c + row));
              sc[c] = fmaf(WIDE ? -sl1 : -sl0, dist, sc[c]);
              if (WIDE) sa[c] = fmaf(-sl0, dist, sa[c]);
            }
          }
          if (!whole) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if ((hidden >> (8 * c + row)) & 1u) {
                sc[c] = -INFINITY;
                if (WIDE) sa[c] = -INFINITY;
              }
            // a row that is not seen has parameters that may be anything: 0 times them has to stay 0
            if ((hidden >> lane) & 1u)
              asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(sb + kLqVMeta + 16 * lane), "r"(0u) : "memory");
            __syncwarp();
          }
        }
        // ---- the values' scales: four tokens of the lane per 16, four groups; their zeros (odd rows of a transposed read)
        uint32_t sv[2][2][4];  // [16 tokens][tokens 2 t4 .. + 1, 2 t4 + 8 ..][group]
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint4 u = lds16(sb + vm_off + 16 * (16 * h + 8 * e)), w = lds16(sb + vm_off + 16 * (16 * h + 8 * e) + 16);
            sv[h][e][0] = lows(u.x, w.x);
            sv[h][e][1] = lows(u.y, w.y);
            sv[h][e][2] = lows(u.z, w.z);
            sv[h][e][3] = lows(u.w, w.w);
          }
        uint32_t zt[4];
        ldsm_x4_t(sb + kLqVMeta + 16 * lane, zt[0], zt[1], zt[2], zt[3]);
        uint32_t lane_top;  // the largest scale of token `lane`
        {
          const uint4 u = lds16(sb + kLqVMeta + 16 * lane);
          lane_top = h2_max(h2_max(u.x, u.y), h2_max(u.z, u.w)) & 0x7fffu;
        }
        // ---- running maximum, and the power of two of the probabilities
        float n1 = max3(fmaxf(sc[0], sc[1]), sc[2], sc[3]), n0 = WIDE ? max3(fmaxf(sa[0], sa[1]), sa[2], sa[3]) : -INFINITY;
        if (__any_sync(0xffffffffu, n1 > m1 || (WIDE && n0 > m0) || lane_top >= scale_top)) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
            if (WIDE) n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, o));
          }
          n1 = fmaxf(n1, m1);
          n0 = fmaxf(n0, m0);
          float f_e = 1.f;
          if (__any_sync(0xffffffffu, lane_top >= scale_top)) {
            const uint32_t t = __reduce_max_sync(0xffffffffu, lane_top);
            const int ex = (int)(t >> 10) - 14;                      // the largest scale is below 2^ex
            const int e = min(max(8 - ex, -8), 15);                  // times 2^e it is below 2^8: seven bits of room above it
            f_e = scale_top == 0 ? 1.f : ex2((float)e - ve);
            scale_top = e < 0 ? 0x8000u : (uint32_t)(30 - e) << 10;  // 2^(15 - e); below e = 0 no scale is too large
            ve = (float)e;
          }
          const float f1 = (n1 == m1 ? 1.f : ex2(m1 - n1)) * f_e, f0 = (n0 == m0 ? 1.f : ex2(m0 - n0)) * f_e;
          m1 = n1;
          m0 = n0;
          l1 *= f1;
          l0 *= f0;
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            acc[c][0] *= WIDE ? f0 : f1;
            acc[c][2] *= WIDE ? f0 : f1;
            if (WIDE) {
              acc[c][1] *= f1;
              acc[c][3] *= f1;
            }
          }
          zacc[0] *= WIDE ? f0 : f1;
          if (WIDE) zacc[1] *= f1;
        }
        if (hidden != 0xffffffffu) {
          const float b1 = m1 == -INFINITY ? 0.f : m1 - ve, b0 = m0 == -INFINITY ? 0.f : m0 - ve;
          uint32_t pb[2][2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float y = ex2(sc[2 * h + e] - b1), x2 = WIDE ? ex2(sa[2 * h + e] - b0) : 0.f;
              l1 += y;
              if (WIDE) l0 += x2;
              pb[h][e] = transpose_8x8(WIDE ? Elem<MC_F16>::pack(x2, y) : Elem<MC_F16>::pack(y, 0.f));
            }
          // ---- D[channel][query row] += codes^T (p scale), zeros^T p
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mma_rows<MC_F16>(zacc, zt[2 * h], zt[2 * h], zt[2 * h + 1], zt[2 * h + 1], pb[h][0], pb[h][1]);
            uint32_t r0[4], r8[4];
            ldsm_x4_t(sb + vc_off + 16 * h * 64, r0[0], r0[1], r0[2], r0[3]);
            ldsm_x4_t(sb + vc_off + (16 * h + 8) * 64, r8[0], r8[1], r8[2], r8[3]);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const uint32_t b0g = h2_mul(pb[h][0], sv[h][0][g]), b8g = h2_mul(pb[h][1], sv[h][1][g]);
              // rows 0..7 of A: a byte, low nibble + 16 high nibble, rows 8..15: 16 high nibble; the difference is taken at the end
              const uint32_t y0 = r0[g] & 0x00ff00ffu, y8 = r8[g] & 0x00ff00ffu;
              const uint32_t w0 = __byte_perm(r0[g], 0, 0x4341), w8 = __byte_perm(r8[g], 0, 0x4341);
              mma_rows<MC_F16>(acc[2 * g], y0, r0[g] & 0x00f000f0u, y8, r8[g] & 0x00f000f0u, b0g, b8g);
              mma_rows<MC_F16>(acc[2 * g + 1], w0, w0 & 0x00f000f0u, w8, w8 & 0x00f000f0u, b0g, b8g);
            }
          }
        }
        if (!whole) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }

      // ---- the piece's result
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l1 += __shfl_xor_sync(0xffffffffu, l1, o);
        if (WIDE) l0 += __shfl_xor_sync(0xffffffffu, l0, o);
      }
      const size_t prow = (size_t)(sh.team + b) * p.n_q_heads + head * nq;
#pragma unroll
      for (int e = 0; e < (WIDE ? 2 : 1); ++e) {
        const int r = WIDE ? 2 * t4 + e : t4;
        float z[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) z[g] = __shfl_sync(0xffffffffu, zacc[e], 4 * (2 * g + 1) + t4);
        if (r >= nq) continue;
        const float m = WIDE && e == 0 ? m0 : m1, l = WIDE && e == 0 ? l0 : l1;
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(p.part_o + (prow + r) * kHeadDim + 32 * g + 4 * row) =
              make_float4(fmaf(acc[2 * g][e] - acc[2 * g][2 + e], 0x1p24f, z[g]), fmaf(acc[2 * g][2 + e], 0x1p20f, z[g]),
                          fmaf(acc[2 * g + 1][e] - acc[2 * g + 1][2 + e], 0x1p24f, z[g]), fmaf(acc[2 * g + 1][2 + e], 0x1p20f, z[g]));
        if (row == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * (prow + r)) = make_float2(m - ve, l);
      }
    }
  }
  if (*s_abort) {  // let copies in flight land before the CTA's memory is released
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
}

// Joins a sequence's pieces (consecutive teams) and its 16-bit rows' part: out = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j.
// A block has R query heads, 8 / R warps each.
constexpr int kLqCombThreads = 256;
constexpr int kLqCombWarps = kLqCombThreads / 32;

template <int DT, int R>
__global__ void __launch_bounds__(kLqCombThreads) layer_q4_combine_kernel(const __grid_constant__ LayerQ4Params p) {
  grid_dep_launch();
  __shared__ float4 acc_s[kLqCombWarps][32];
  __shared__ float l_s[kLqCombWarps], m_s[kLqCombWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.y;
  constexpr int GP = kLqCombWarps / R;  // warps per output row
  const int grp = warp % GP;
  const int hq = blockIdx.x * R + warp / GP;
  const bool active = hq < p.n_q_heads;
  grid_dep_wait();
  const int4 pc = __ldcg(p.pieces + b);
  const int c0 = pc.x, n_pages = pc.y, begun = pc.z;
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (active) {
    const int n_parts = n_pages + begun;
    for (int c = grp; c < n_parts; c += 4 * GP) {  // four parts in flight
      float2 ml[4];
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        const int j = c + k * GP;
        if (j < n_parts) {
          const size_t prow = j < n_pages ? (size_t)(c0 + j + b) * p.n_q_heads + hq : (size_t)p.res_part + (size_t)b * p.n_q_heads + hq;
          ml[k] = *reinterpret_cast<const float2*>(p.part_ml + 2 * prow);
          v[k] = *reinterpret_cast<const float4*>(p.part_o + prow * kHeadDim + 4 * lane);
        }
      }
      float M2 = M;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (ml[k].y != 0.f) M2 = fmaxf(M2, ml[k].x);
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
    acc_s[warp][lane] = o;
    if (lane == 0) {
      l_s[warp] = L;
      m_s[warp] = M;
    }
    __syncthreads();
    if (grp != 0 || !active) return;
    float Ma = M;
    for (int g = 1; g < GP; ++g) Ma = fmaxf(Ma, m_s[warp + g]);
    const float f = L == 0.f ? 0.f : ex2(M - Ma);
    L *= f;
    o.x *= f;
    o.y *= f;
    o.z *= f;
    o.w *= f;
    for (int g = 1; g < GP; ++g) {
      const float lg = l_s[warp + g], fg = lg == 0.f ? 0.f : ex2(m_s[warp + g] - Ma);
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
  *reinterpret_cast<uint2*>(p.out + orow * kHeadDim + lane * 4) = packed;
  if (lane == 0 && p.lse != nullptr) p.lse[orow] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

// ---- host side ------------------------------------------------------------------------------------
struct LayerQ4Plan {
  int members, n_teams;
  long long max_units;
  size_t rows, o_bytes, ml_bytes, piece_bytes;
};
// The workspace is sized for kLqMaxCtas CTAs, so that its size needs no device.
constexpr int kLqMaxCtas = 512;
static LayerQ4Plan layer_q4_plan(const mc_config* cfg, const mc_batch* bt, int ctas) {
  LayerQ4Plan pl;
  const int warps = std::min(ctas, kLqMaxCtas) * kLqWarps;
  const int per_warp = (cfg->n_kv_heads + warps - 1) / warps;  // heads
  pl.members = (cfg->n_kv_heads + per_warp - 1) / per_warp;
  pl.max_units = (long long)bt->batch * (bt->max_seq_len / kLqPage + kLqBegunUnits);
  pl.n_teams = (int)std::max<long long>(1, std::min<long long>(warps / pl.members, pl.max_units));
  pl.rows = (size_t)(pl.n_teams + bt->batch) * cfg->n_q_heads + (size_t)bt->batch * cfg->n_q_heads;
  pl.o_bytes = align_up(pl.rows * kHeadDim * 4, 256);
  pl.ml_bytes = align_up(pl.rows * 2 * 4, 256);
  pl.piece_bytes = align_up((size_t)bt->batch * sizeof(int4), 256);
  return pl;
}
static constexpr size_t q4_smem_bytes(int batch) {
  return 1024 + (size_t)kLqWarps * kLqStages * (kLqStageBytes + 8) + (size_t)(batch + 2) * (8 + sizeof(Q4Seq));
}
static_assert(q4_smem_bytes(kMaxLayerBatch) <= 227 * 1024, "a CTA's shared memory");

size_t layer_q4_attn_workspace_bytes(const mc_config* cfg, const mc_batch* bt, int) {
  const LayerQ4Plan pl = layer_q4_plan(cfg, bt, kLqMaxCtas);
  return pl.o_bytes + pl.ml_bytes + pl.piece_bytes;
}

mc_status launch_layer_q4_attn(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer,
                               const mc_score_opts* opts, const int32_t* pages, const int32_t* counts, int pages_stride, const void* q,
                               const void* k_new, const void* v_new, int flags, void* out, float* lse, void* workspace,
                               cudaStream_t stream) {
  if (bt->batch == 0) return MC_OK;
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  const int ctas = std::min(n_sm * kLqCtasPerSm, kLqMaxCtas);
  const LayerQ4Plan pl = layer_q4_plan(cfg, bt, ctas);
  CUtensorMap map_km, map_vc;
  const uint64_t tiles = (uint64_t)std::max<int64_t>(bt->n_pages, 1) * cfg->n_kv_heads;
  if (mc_status st = make_map_rows(&map_km, layer->k_meta, tiles * 4, 128, 4)) return st;
  if (mc_status st = make_map_rows(&map_vc, layer->v_codes, tiles * kLqPage, 64, kLqPage)) return st;
  LayerQ4Params ap;
  ap.g = g;
  ap.rule = make_score_rule(opts);
  ap.k_codes = (const unsigned char*)layer->k_codes;
  ap.v_meta = (const unsigned char*)layer->v_meta;
  ap.pool[0] = (unsigned char*)layer->k_codes;
  ap.pool[1] = (unsigned char*)layer->k_meta;
  ap.pool[2] = (unsigned char*)layer->v_codes;
  ap.pool[3] = (unsigned char*)layer->v_meta;
  ap.res_k = (char*)layer->res_k;
  ap.res_v = (char*)layer->res_v;
  ap.status = layer->status;
  ap.q = (const char*)q;
  ap.k_new = (const char*)k_new;
  ap.v_new = (const char*)v_new;
  ap.sel = pages;
  ap.counts = counts;
  ap.sel_stride = pages_stride;
  ap.part_o = (float*)workspace;
  ap.part_ml = (float*)((char*)workspace + pl.o_bytes);
  ap.pieces = (int4*)((char*)workspace + pl.o_bytes + pl.ml_bytes);
  ap.nq = cfg->n_q_heads / cfg->n_kv_heads;
  ap.n_q_heads = cfg->n_q_heads;
  ap.members = pl.members;
  ap.n_teams = pl.n_teams;
  ap.res_part = (pl.n_teams + bt->batch) * cfg->n_q_heads;
  ap.flags = flags;
  ap.out = (unsigned short*)out;
  ap.lse = lse;
  const bool wide = ap.nq == 8;
  auto* split = cfg->dtype == MC_F16 ? (wide ? layer_q4_split_kernel<MC_F16, true> : layer_q4_split_kernel<MC_F16, false>)
                                     : (wide ? layer_q4_split_kernel<MC_BF16, true> : layer_q4_split_kernel<MC_BF16, false>);
  MC_CUDA_CHECK(allow_smem(split, q4_smem_bytes(kMaxLayerBatch)));
  const int grid = (pl.n_teams * pl.members + kLqWarps - 1) / kLqWarps;
  MC_CUDA_CHECK(launch_pdl(split, dim3(grid), dim3(kLqThreads), q4_smem_bytes(bt->batch), stream, ap, map_km, map_vc));
  // warps per output row: about three parts each
  const long long parts = pl.n_teams / bt->batch + 2;
  int per_block = kLqCombWarps;  // rows
  while (per_block > 1 && parts > 3 * (kLqCombWarps / per_block)) per_block /= 2;
  using Combine = void (*)(const LayerQ4Params);
  static const Combine combines[2][4] = {
      {layer_q4_combine_kernel<MC_F16, 1>, layer_q4_combine_kernel<MC_F16, 2>, layer_q4_combine_kernel<MC_F16, 4>,
       layer_q4_combine_kernel<MC_F16, 8>},
      {layer_q4_combine_kernel<MC_BF16, 1>, layer_q4_combine_kernel<MC_BF16, 2>, layer_q4_combine_kernel<MC_BF16, 4>,
       layer_q4_combine_kernel<MC_BF16, 8>}};
  const Combine combine = combines[cfg->dtype == MC_F16 ? 0 : 1][per_block == 1 ? 0 : per_block == 2 ? 1 : per_block == 4 ? 2 : 3];
  MC_CUDA_CHECK(launch_pdl(combine, dim3((cfg->n_q_heads + per_block - 1) / per_block, bt->batch), dim3(kLqCombThreads), 0, stream, ap));
  MC_CUDA_CHECK(cudaGetLastError());
  return MC_OK;
}

}  // namespace mc
