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
// A sequence's complete pages as a query sees them: tokens [0, a) and [lo, hi), so the pages [0, ua) and those from ub0
// on, u in all.
struct PageView {
  int n;             // cached tokens
  int q_pos;
  int a, lo, hi;
  int ua, ub0, u;
  __device__ __forceinline__ int page_of(int k) const { return k < ua ? k : ub0 + k - ua; }
  __device__ __forceinline__ bool sees(int t) const { return t < a || (t >= lo && t < hi); }
  __device__ __forceinline__ bool all_of(int t0) const { return t0 + kLqPage <= a || (t0 >= lo && t0 + kLqPage <= hi); }
  __device__ __forceinline__ bool some_of(int t0) const { return t0 < a || (t0 + kLqPage > lo && t0 < hi); }
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
  const int full = n / kLqPage * kLqPage;  // tokens in complete pages
  const int a = min(s.a, full), hi = min(s.hi, full);
  s.ua = (a + kLqPage - 1) / kLqPage;
  s.ub0 = max(s.lo / kLqPage, s.ua);
  const int ub1 = hi > s.lo ? (hi + kLqPage - 1) / kLqPage : 0;
  s.u = s.ua + max(ub1 - s.ub0, 0);
  return s;
}

// Exclusive prefix of [0, batch) counts in shared memory, pre[b + 1] = the count of sequence b on entry; pre[batch] = the
// total.  Every thread of the CTA calls it.
__device__ __forceinline__ void scan_counts(int* pre, int batch) {
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, per = (batch + 31) / 32;
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
__device__ __forceinline__ uint2 lq_tame(const uint2& r) {
  const float2 a = Elem<DT>::unpack(r.x), b = Elem<DT>::unpack(r.y);
  return make_uint2(Elem<DT>::pack(lq_tame<DT>(a.x), lq_tame<DT>(a.y)), Elem<DT>::pack(lq_tame<DT>(b.x), lq_tame<DT>(b.y)));
}
// Two numbers of a word less z: for binary16 one mixed-precision FMA each.
template <int DT>
__device__ __forceinline__ float2 minus(uint32_t w, float zx, float zy) {
  if (DT == MC_F16) {
    float2 r;
    asm("{\n\t.reg .b16 lo, hi, one;\n\tmov.b32 {lo, hi}, %2;\n\tmov.b16 one, 0x3C00;\n\t"
        "fma.rn.f32.f16 %0, lo, one, %3;\n\tfma.rn.f32.f16 %1, hi, one, %4;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "r"(w), "f"(-zx), "f"(-zy));
    return r;
  }
  const float2 v = Elem<DT>::unpack(w);
  return make_float2(v.x - zx, v.y - zy);
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Four codes, channel 4l + j at bits 4j, of differences d with scales' reciprocals inv, for quotients between 0 and 15.01; `tie`: one
// of them is next to a tie (they are at most 15 * 3 * 2^-24 off).
__device__ __forceinline__ uint32_t lq_codes(const float (&d)[4], const float (&inv)[4], bool& tie) {
  float r[4], e[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    r[j] = fmaf(d[j], inv[j], 12582912.0f) - 12582912.0f;  // 1.5 * 2^23: the nearest integer
    e[j] = fmaf(d[j], inv[j], -r[j]);
  }
  tie = max3_abs(fmaxf(fabsf(e[0]), fabsf(e[1])), e[2], e[3]) > 0.49999f;
  return (uint32_t)__float_as_int(fmaf(fmaf(r[3], 16.f, r[2]), 256.f, fmaf(r[1], 16.f, r[0])) + 12582912.0f) & 0xffffu;
}
template <int DT>
__device__ __forceinline__ uint32_t lq_codes_exact(const uint2& r, const float (&z)[4], const float (&s)[4]) {
  const float2 a = Elem<DT>::unpack(r.x), b = Elem<DT>::unpack(r.y);
  const float x[4] = {a.x, a.y, b.x, b.y};
  uint32_t c = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) c |= (uint32_t)lq_code(x[j], z[j], s[j], 1.0f / s[j]) << (4 * j);
  return c;
}
// A group whose quotients may leave [0, 15.01]: a scale that is subnormal (coarse), a zero that is not the minimum itself.
__device__ __forceinline__ bool lq_odd(uint32_t group, float lo) { return (group & 0x7fffu) < 0x0400u || half_hi(group) != lo; }

// One (page, kv head) of K or V by a warp: lane l has channels 4l .. 4l + 3 of the page's 32 rows, load(t) gives those of row t.
// False (nothing stored that counts): something in it is not a number that binary16 holds, and it has to be done again with WILD.
// Loops that are not unrolled over registers: 16 KB of straight code per tensor made the instruction cache the limit (8 x 4096
// prompts of 32 heads 606 us).
// K: a group is one of the lane's channels, so nothing is exchanged.
template <int DT, bool WILD, typename Load>
__device__ __forceinline__ bool lq_quantise_keys(Load load, unsigned char* codes, unsigned char* meta) {
  const int lane = threadIdx.x & 31;
  auto get = [&](int t) { return WILD ? lq_tame<DT>(load(t)) : load(t); };
  uint2 lo2 = get(0), hi2 = lo2;
#pragma unroll 8
  for (int t = 1; t < kLqPage; ++t) {
    const uint2 r = get(t);
    lo2.x = min2_nan<DT>(lo2.x, r.x);
    lo2.y = min2_nan<DT>(lo2.y, r.y);
    hi2.x = max2_nan<DT>(hi2.x, r.x);
    hi2.y = max2_nan<DT>(hi2.y, r.y);
  }
  const float2 la = Elem<DT>::unpack(lo2.x), lb = Elem<DT>::unpack(lo2.y), ha = Elem<DT>::unpack(hi2.x), hb = Elem<DT>::unpack(hi2.y);
  const float lo[4] = {la.x, la.y, lb.x, lb.y}, hi[4] = {ha.x, ha.y, hb.x, hb.y};
  if (!WILD) {
    bool tame = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) tame = tame && lo[j] >= -65504.f && hi[j] <= 65504.f;  // (false for a NaN)
    if (!__all_sync(0xffffffffu, tame)) return false;
  }
  uint32_t w[4];
  float z[4], s[4], inv[4];
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] = lq_group(lo[j], hi[j]);
    s[j] = half_lo(w[j]);
    z[j] = half_hi(w[j]);
    inv[j] = rcp_approx(s[j]);
    odd = odd || lq_odd(w[j], lo[j]);
  }
  *reinterpret_cast<uint4*>(meta + 16 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
  unsigned short* out = reinterpret_cast<unsigned short*>(codes) + lane;
  uint32_t again = 0;  // rows with a quotient next to a tie
#pragma unroll 4
  for (int t = 0; t < kLqPage; ++t) {
    const uint2 r = get(t);
    const float2 a = minus<DT>(r.x, z[0], z[1]), b = minus<DT>(r.y, z[2], z[3]);
    const float d[4] = {a.x, a.y, b.x, b.y};
    bool tie;
    out[32 * t] = (unsigned short)lq_codes(d, inv, tie);
    if (tie) again |= 1u << t;
  }
  again = __any_sync(0xffffffffu, odd) ? 0xffffffffu : __reduce_or_sync(0xffffffffu, again);
#pragma unroll 1
  while (again != 0) {
    const int t = __ffs(again) - 1;
    again &= again - 1;
    out[32 * t] = (unsigned short)lq_codes_exact<DT>(get(t), z, s);
  }
  return true;
}
// V: a group is a row's part in eight lanes.  Eight rows' extremes (the least and the negative of the largest, a pair) are joined
// at a time, halving the rows a lane keeps at every step (7 exchanges instead of 24); lane j of the eight ends with row j's
// group, forms its parameters once and hands them round.
template <int DT, bool WILD, typename Load>
__device__ __forceinline__ bool lq_quantise_values(Load load, unsigned char* codes, unsigned char* meta) {
  const int lane = threadIdx.x & 31, j8 = lane & 7;
  auto get = [&](int t) { return WILD ? lq_tame<DT>(load(t)) : load(t); };
  unsigned short* out = reinterpret_cast<unsigned short*>(codes) + lane;
#pragma unroll 1
  for (int t0 = 0; t0 < kLqPage; t0 += 8) {
    uint2 r[8];
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      r[i] = get(t0 + i);
      const uint32_t mn = min2_nan<DT>(r[i].x, r[i].y), mx = max2_nan<DT>(r[i].x, r[i].y) ^ 0x80008000u;
      v[i] = min2_nan<DT>(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
    }
#pragma unroll
    for (int o = 4, m = 4; o > 0; o >>= 1, m >>= 1) {  // m rows stay: those whose bit o is the lane's
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
    *reinterpret_cast<uint32_t*>(meta + 16 * (t0 + j8) + 4 * (lane >> 3)) = own;
    uint32_t again = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w = __shfl_sync(0xffffffffu, own, (lane & 24) + i);
      const float f = __shfl_sync(0xffffffffu, own_inv, (lane & 24) + i), z = half_hi(w);
      const float2 a = minus<DT>(r[i].x, z, z), b = minus<DT>(r[i].y, z, z);
      const float d[4] = {a.x, a.y, b.x, b.y}, inv[4] = {f, f, f, f};
      bool tie;
      out[32 * (t0 + i)] = (unsigned short)lq_codes(d, inv, tie);
      if (tie) again |= 1u << i;
    }
    again = __any_sync(0xffffffffu, lq_odd(own, lo)) ? 0xffu : __reduce_or_sync(0xffffffffu, again);
#pragma unroll 1
    while (again != 0) {
      const int i = __ffs(again) - 1;
      again &= again - 1;
      const uint32_t w = __shfl_sync(0xffffffffu, own, (lane & 24) + i);
      const float s = half_lo(w), z = half_hi(w);
      const float s4[4] = {s, s, s, s}, z4[4] = {z, z, z, z};
      out[32 * (t0 + i)] = (unsigned short)lq_codes_exact<DT>(get(t0 + i), z4, s4);
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
