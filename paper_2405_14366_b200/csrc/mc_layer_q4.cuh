// Device pieces shared by the operators of a layer held in 4 bits (mc_layer_q4 pools: keys per channel over a page of
// 32 tokens, values per token over 32 channels): tile sizes, what a query sees in pages, the quantiser of a page.
#pragma once
#include "mc_layer.cuh"

namespace mc {

constexpr int kLqPage = 32;                        // tokens per page: a key group
constexpr int kLqCodeBytes = kLqPage * 64;         // codes of one (page, kv head), K or V
constexpr int kLqMetaBytes = 512;                  // (scale, zero): K [128], V [32][4]
constexpr int kLqResBytes = kLqPage * kRowBytes;   // the begun page's rows of one (sequence, kv head)

#if defined(__CUDACC__)
// A sequence as a query sees it: the tokens [0, a) and [lo, hi).
struct TokenView {
  int n;  // cached tokens
  int q_pos;
  int a, lo, hi;
  __device__ __forceinline__ int full() const { return n / kLqPage; }  // complete pages
  __device__ __forceinline__ bool sees(int t) const { return t < a || (t >= lo && t < hi); }
  __device__ __forceinline__ bool all_of(int t0) const { return t0 + kLqPage <= a || (t0 >= lo && t0 + kLqPage <= hi); }
  // the complete pages with a token that is seen: [0, head_pages) and those from tail_page on
  __device__ __forceinline__ int head_pages() const { return (min(a, full() * kLqPage) + kLqPage - 1) / kLqPage; }
  __device__ __forceinline__ int tail_page(int head) const { return max(lo / kLqPage, head); }
};
// The same with these pages, u in all: [0, ua) and those from ub0 on.
struct PageView : TokenView {
  int ua, ub0, u;
  __device__ __forceinline__ int page_of(int k) const { return k < ua ? k : ub0 + k - ua; }
};
// n_tot: tokens that count for the masks, the step's new one included; default_pos: the query's position without q_pos.
__device__ __forceinline__ PageView page_view(const ScoreRule& rule, int b, int n, int n_tot, int default_pos) {
  PageView s;
  const View v = view_at(rule, b, max(rule.q_pos ? rule.q_pos[b] : default_pos, -1));
  s.n = n;
  s.q_pos = v.q_pos;
  const int end = min(n_tot - 1, v.q_pos) + 1;  // one past the last token the query may see
  s.a = max(min(end, v.prefix), 0);
  s.lo = max(v.lo_pos, s.a);
  s.hi = max(end, s.lo);
  s.ua = s.head_pages();
  s.ub0 = s.tail_page(s.ua);
  const int hi = min(s.hi, s.full() * kLqPage);
  const int ub1 = hi > s.lo ? (hi + kLqPage - 1) / kLqPage : 0;
  s.u = s.ua + max(ub1 - s.ub0, 0);
  return s;
}

// Exclusive prefix of counts in shared memory by a warp: pre[b + 1] = the count of sequence b on entry; pre[batch] = the total.
__device__ __forceinline__ void scan_warp(int* pre, int batch) {
  const int lane = threadIdx.x & 31, per = (batch + 31) / 32;
  const int b0 = min(lane * per, batch), b1 = min(b0 + per, batch);
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
// The same for a CTA: every thread calls it.
__device__ __forceinline__ void scan_counts(int* pre, int batch) {
  __syncthreads();
  if (threadIdx.x < 32) scan_warp(pre, batch);
  __syncthreads();
}
__device__ __forceinline__ int seq_of_item(const int* pre, int batch, int x) {
  int lo = 0, hi = batch - 1;  // last b with pre[b] <= x
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ---- the quantiser ---------------------------------------------------------------------------------------
// Both roundings below are those of the exact quotient.  They are made in binary32, where a quotient is a few units of the
// last place off, and looked at again where it comes next to a tie: the difference of two numbers is d + e exactly (Knuth's
// two-term sum), a multiple of a 16-bit number by a small one is exact, and so is what is left of d next to that multiple;
// the sign of the rest plus e decides.  (64-bit arithmetic in its place cost the kernel 750 bytes of spilled registers.)
__device__ __forceinline__ float diff_error(float x, float z, float d) {  // x - z = d + this
  const float bb = d - x;
  return (x - (d - bb)) - (z + bb);
}
// code = clamp(rint((x - zero) / scale), 0, 15): ties to even.
__device__ __forceinline__ int lq_code(float x, float z, float s, float inv_s) {
  const float d = x - z;
  const float q = fminf(fmaxf(d * inv_s, 0.f), 15.f);  // (at most 15 * 4 * 2^-24 off)
  const float m = q + 12582912.0f;                     // 1.5 * 2^23: rint(q) in the last bits
  int c = __float_as_int(m) & 15;
  if (fabsf(q - (m - 12582912.0f)) > 0.4999f) {
    const float k = floorf(q), rest = fmaf(-(k + 0.5f), s, d) + diff_error(x, z, d);
    c = (int)k;
    c += rest > 0.f ? 1 : rest == 0.f ? (c & 1) : 0;
  }
  return c;
}
// (scale, zero) of a group from its extremes, in one word as the pools hold it: scale = half((hi - lo) / 15).
__device__ __forceinline__ uint32_t lq_group(float lo, float hi) {
  const float d = fabsf(hi - lo);  // (-0 where the largest came as -0)
  uint32_t s = __half_as_ushort(__float2half_rd(d * (1.0f / 15.0f)));  // the number below (or one too low, next to a number)
  const float a = __half2float(__ushort_as_half((unsigned short)s)), b = __half2float(__ushort_as_half((unsigned short)(s + 1)));
  const float rest = fmaf(-7.5f, a + b, d) + diff_error(hi, lo, d);  // against 15 times the middle
  s += rest > 0.f ? 1u : rest == 0.f ? (s & 1u) : 0u;
  if (s == 0) s = 0x3C00;  // a constant group: scale 1
  const uint32_t z = __half_as_ushort(__float2half_rn(lo));
  return s | ((z & 0x7fffu) == 0 ? 0u : z << 16);  // (which of two zeros is the least is nobody's business: +0)
}
__device__ __forceinline__ float half_lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
__device__ __forceinline__ float half_hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
// Element by element of a pair of 16-bit numbers, a NaN if either is one.
template <int DT>
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  if (DT == MC_F16) asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int DT>
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  if (DT == MC_F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// What a page takes in: what binary16 can hold (the largest bfloat16 below 65504 is 65280), a NaN as 0.
template <int DT>
__device__ __forceinline__ float lq_tame(float x) {
  constexpr float most = DT == MC_F16 ? 65504.f : 65280.f;
  return x != x ? 0.f : fminf(fmaxf(x, -most), most);
}
template <int DT>
__device__ __forceinline__ uint32_t lq_tame2(uint32_t w) {
  const float2 a = Elem<DT>::unpack(w);
  return Elem<DT>::pack(lq_tame<DT>(a.x), lq_tame<DT>(a.y));
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two numbers of a word less z (nz = -z, two numbers): for binary16 one mixed-precision FMA each.
template <int DT>
__device__ __forceinline__ uint64_t plus2(uint32_t w, uint64_t nz) {
  float zx, zy;
  unpack2(nz, zx, zy);
  if (DT == MC_F16) {
    float x, y;
    asm("{\n\t.reg .b16 lo, hi, one;\n\tmov.b32 {lo, hi}, %2;\n\tmov.b16 one, 0x3C00;\n\t"
        "fma.rn.f32.f16 %0, lo, one, %3;\n\tfma.rn.f32.f16 %1, hi, one, %4;\n\t}"
        : "=f"(x), "=f"(y)
        : "r"(w), "f"(zx), "f"(zy));
    return pack2(x, y);
  }
  const float2 v = Elem<DT>::unpack(w);
  return add2(pack2(v.x, v.y), nz);
}
// The codes of eight channels of a row, channel j at bits 4j, for quotients between 0 and 15.01; `tie`: one of them is next to a
// tie (they are at most 15 * 3 * 2^-24 off).  nz, inv: -zero and 1 / scale of channel pairs.  Two channels per instruction.
template <int DT>
__device__ __forceinline__ uint32_t lq_codes(const uint4& r, const uint64_t (&nz)[4], const uint64_t (&inv)[4], bool& tie) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  const uint64_t magic = pack2(12582912.0f, 12582912.0f), minus1 = pack2(-1.f, -1.f);  // 1.5 * 2^23: the nearest integer
  float c[8], worst = 0.f;  // c: codes' negatives
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t d = plus2<DT>(w[j], nz[j]);
    const uint64_t n = fma2(fma2(d, inv[j], magic), minus1, magic);
    float ex, ey;
    unpack2(fma2(d, inv[j], n), ex, ey);
    worst = max3_abs(worst, ex, ey);
    unpack2(n, c[2 * j], c[2 * j + 1]);
  }
  tie = worst > 0.49999f;
  const float lo = 12582912.0f - fmaf(fmaf(c[3], 16.f, c[2]), 256.f, fmaf(c[1], 16.f, c[0]));
  const float hi = 12582912.0f - fmaf(fmaf(c[7], 16.f, c[6]), 256.f, fmaf(c[5], 16.f, c[4]));
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
}
// The same, every code for itself and right whatever the quotient is; group(j): (scale, zero) of channel j.
template <int DT, typename Group>
__device__ __forceinline__ uint32_t lq_codes_exact(const uint4& r, Group group) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  uint32_t c = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 x = Elem<DT>::unpack(w[j >> 1]);
    const uint32_t g = group(j);
    const float s = half_lo(g);
    c |= (uint32_t)lq_code(j & 1 ? x.y : x.x, half_hi(g), s, rcp_approx(s)) << (4 * j);
  }
  return c;
}
// A group whose quotients may leave [0, 15.01]: a scale that is subnormal (coarse), a zero that is not the minimum itself.
__device__ __forceinline__ bool lq_odd(uint32_t group, float lo) { return (group & 0x7fffu) < 0x0400u || half_hi(group) != lo; }

// One (page, kv head) of K or V by a warp: half a warp has a row, lane l channels 8 (l & 15) .. + 7 of the rows 2k + (l >> 4);
// load(t) gives those of row t.  False (nothing stored that counts): something in it is not a number that binary16 holds, and it
// has to be done again with WILD.  The rows come from memory, not from registers: with a page in registers the code was 16 KB of
// straight lines per tensor and the instruction cache the limit (8 x 4096 prompts of 32 heads 606 us).
// K: a group is one of the lane's channels; the two half-warps join their extremes.
template <int DT, bool WILD, typename Load>
__device__ __forceinline__ bool lq_quantise_keys(Load load, unsigned char* codes, unsigned char* meta) {
  const int lane = threadIdx.x & 31, half = lane >> 4, ch = lane & 15;
  auto get = [&](int k) {
    uint4 r = load(2 * k + half);
    if (WILD) r = make_uint4(lq_tame2<DT>(r.x), lq_tame2<DT>(r.y), lq_tame2<DT>(r.z), lq_tame2<DT>(r.w));
    return r;
  };
  uint32_t lo2[4], hi2[4];
  {
    const uint4 r = get(0);
    lo2[0] = hi2[0] = r.x;
    lo2[1] = hi2[1] = r.y;
    lo2[2] = hi2[2] = r.z;
    lo2[3] = hi2[3] = r.w;
  }
#pragma unroll 5
  for (int k = 1; k < kLqPage / 2; ++k) {
    const uint4 r = get(k);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo2[j] = min2_nan<DT>(lo2[j], w[j]);
      hi2[j] = max2_nan<DT>(hi2[j], w[j]);
    }
  }
  bool tame = true, odd = false;
  uint32_t own[4], group[8];  // a half-warp forms the parameters of four of a lane's channels, the other half those of the others
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    // (the other half's extremes of the channels that are this lane's to do, for this half's of the others)
    const uint32_t gl = half ? lo2[j] : lo2[j + 2], gh = half ? hi2[j] : hi2[j + 2], kl = half ? lo2[j + 2] : lo2[j], kh = half ? hi2[j + 2] : hi2[j];
    const float2 lo = Elem<DT>::unpack(min2_nan<DT>(kl, __shfl_xor_sync(0xffffffffu, gl, 16)));
    const float2 hi = Elem<DT>::unpack(max2_nan<DT>(kh, __shfl_xor_sync(0xffffffffu, gh, 16)));
    tame = tame && lo.x >= -65504.f && lo.y >= -65504.f && hi.x <= 65504.f && hi.y <= 65504.f;  // (false for a NaN)
    own[2 * j] = lq_group(lo.x, hi.x);
    own[2 * j + 1] = lq_group(lo.y, hi.y);
    odd = odd || lq_odd(own[2 * j], lo.x) || lq_odd(own[2 * j + 1], lo.y);
  }
  if (!WILD && !__all_sync(0xffffffffu, tame)) return false;
  *reinterpret_cast<uint4*>(meta + 32 * ch + 16 * half) = make_uint4(own[0], own[1], own[2], own[3]);
  uint64_t nz[4], inv[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, own[j], 16);
    group[j] = half ? other : own[j];
    group[j + 4] = half ? own[j] : other;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    nz[j] = pack2(-half_hi(group[2 * j]), -half_hi(group[2 * j + 1]));
    inv[j] = pack2(rcp_approx(half_lo(group[2 * j])), rcp_approx(half_lo(group[2 * j + 1])));
  }
  uint32_t* out = reinterpret_cast<uint32_t*>(codes) + lane;
  uint32_t again = 0;  // row pairs with a quotient next to a tie
#pragma unroll 4
  for (int k = 0; k < kLqPage / 2; ++k) {
    bool tie;
    out[32 * k] = lq_codes<DT>(get(k), nz, inv, tie);
    if (tie) again |= 1u << k;
  }
  again = __any_sync(0xffffffffu, odd) ? 0xffffu : __reduce_or_sync(0xffffffffu, again);
#pragma unroll 1
  while (again != 0) {
    const int k = __ffs(again) - 1;
    again &= again - 1;
    out[32 * k] = lq_codes_exact<DT>(get(k), [&](int j) { return group[j]; });
  }
  return true;
}
// V: a group is a row's part in four lanes.  The extremes of a lane's four rows (the least and the negative of the largest, a pair)
// are joined at a time, halving the rows that a lane keeps (3 exchanges instead of 8); lane j of the four ends with row j's
// group, forms its parameters once and hands them round.
template <int DT, bool WILD, typename Load>
__device__ __forceinline__ bool lq_quantise_values(Load load, unsigned char* codes, unsigned char* meta) {
  const int lane = threadIdx.x & 31, half = lane >> 4, ch = lane & 15;
  auto get = [&](int k) {
    uint4 r = load(2 * k + half);
    if (WILD) r = make_uint4(lq_tame2<DT>(r.x), lq_tame2<DT>(r.y), lq_tame2<DT>(r.z), lq_tame2<DT>(r.w));
    return r;
  };
  uint32_t* out = reinterpret_cast<uint32_t*>(codes) + lane;
#pragma unroll 1
  for (int k0 = 0; k0 < kLqPage / 2; k0 += 4) {
    uint4 r[4];
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = get(k0 + i);
      const uint32_t mn = min2_nan<DT>(min2_nan<DT>(r[i].x, r[i].y), min2_nan<DT>(r[i].z, r[i].w));
      const uint32_t mx = max2_nan<DT>(max2_nan<DT>(r[i].x, r[i].y), max2_nan<DT>(r[i].z, r[i].w)) ^ 0x80008000u;
      v[i] = min2_nan<DT>(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
    }
#pragma unroll
    for (int o = 2, m = 2; o > 0; o >>= 1, m >>= 1) {  // m rows stay: those whose bit o is the lane's
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < m; ++i) {
        const uint32_t give = up ? v[i] : v[i + m], keep = up ? v[i + m] : v[i];
        v[i] = min2_nan<DT>(keep, __shfl_xor_sync(0xffffffffu, give, o));
      }
    }
    const float2 mm = Elem<DT>::unpack(v[0]);
    const float lo = mm.x, hi = -mm.y;
    if (!WILD && !__all_sync(0xffffffffu, lo >= -65504.f && hi <= 65504.f)) return false;
    const uint32_t own = lq_group(lo, hi);
    const float own_inv = rcp_approx(half_lo(own));
    *reinterpret_cast<uint32_t*>(meta + 16 * (2 * (k0 + (lane & 3)) + half) + 4 * (ch >> 2)) = own;
    uint32_t again = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float z = -half_hi(__shfl_sync(0xffffffffu, own, (lane & 28) + i)), f = __shfl_sync(0xffffffffu, own_inv, (lane & 28) + i);
      const uint64_t z2 = pack2(z, z), f2 = pack2(f, f);
      const uint64_t nz[4] = {z2, z2, z2, z2}, inv[4] = {f2, f2, f2, f2};
      bool tie;
      out[32 * (k0 + i)] = lq_codes<DT>(r[i], nz, inv, tie);
      if (tie) again |= 1u << i;
    }
    again = __any_sync(0xffffffffu, lq_odd(own, lo)) ? 0xfu : __reduce_or_sync(0xffffffffu, again);
#pragma unroll 1
    while (again != 0) {
      const int i = __ffs(again) - 1;
      again &= again - 1;
      const uint32_t w = __shfl_sync(0xffffffffu, own, (lane & 28) + i);
      out[32 * (k0 + i)] = lq_codes_exact<DT>(get(k0 + i), [&](int) { return w; });
    }
  }
  return true;
}
template <int DT, typename Load>
__device__ __forceinline__ void lq_quantise(bool keys, Load load, unsigned char* codes, unsigned char* meta) {
  if (keys) {
    if (!lq_quantise_keys<DT, false>(load, codes, meta)) lq_quantise_keys<DT, true>(load, codes, meta);
  } else {
    if (!lq_quantise_values<DT, false>(load, codes, meta)) lq_quantise_values<DT, true>(load, codes, meta);
  }
}
#endif

}  // namespace mc
