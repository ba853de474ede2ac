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
  const float d = hi - lo;
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
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// What a page takes in: what binary16 can hold (the largest bfloat16 below 65504 is 65280), a NaN as 0.
template <int DT>
__device__ __forceinline__ float lq_tame(float x) {
  constexpr float most = DT == MC_F16 ? 65504.f : 65280.f;
  return x != x ? 0.f : fminf(fmaxf(x, -most), most);
}
template <int DT>
__device__ __forceinline__ void lq_tame_words(uint2 (&r)[kLqPage]) {
#pragma unroll
  for (int t = 0; t < kLqPage; ++t) {
    asm volatile("" : "+r"(r[t].x), "+r"(r[t].y));  // (row by row: see `four` below)
    const float2 a = Elem<DT>::unpack(r[t].x), b = Elem<DT>::unpack(r[t].y);
    r[t].x = Elem<DT>::pack(lq_tame<DT>(a.x), lq_tame<DT>(a.y));
    r[t].y = Elem<DT>::pack(lq_tame<DT>(b.x), lq_tame<DT>(b.y));
  }
}

// (in program order: a row's codes leave before the next row's are worked out)
__device__ __forceinline__ void st_code(unsigned short* p, uint32_t c) {
  asm volatile("st.global.u16 [%0], %1;" ::"l"(p), "h"((unsigned short)c) : "memory");
}

// One (page, kv head) of K or V by a warp: lane l holds channels 4l .. 4l + 3 of the page's 32 rows.
// K: a group is one of the lane's channels, so nothing is exchanged.  V: a group is a row's part in eight lanes; eight
// rows' extremes are joined at a time, halving the rows a lane keeps at every step (7 exchanges instead of 24), so that lane
// j of the eight ends with row j's group, forms its parameters once and hands them round.
template <int DT>
__device__ __forceinline__ void lq_quantise(bool keys, uint2 (&r)[kLqPage], unsigned char* codes, unsigned char* meta) {
  const int lane = threadIdx.x & 31;
  const float inf = __int_as_float(0x7f800000);
  // (the words pass through an empty statement every time: the compiler would keep all 128 numbers of the first pass, in
  // local memory, for the second)
  auto four = [&](int t, float (&x)[4]) {
    asm volatile("" : "+r"(r[t].x), "+r"(r[t].y));
    const float2 a = Elem<DT>::unpack(r[t].x), b = Elem<DT>::unpack(r[t].y);
    x[0] = a.x;
    x[1] = a.y;
    x[2] = b.x;
    x[3] = b.y;
  };
  float lo[4], hi[4];
#pragma unroll 1
  for (int again = 0; again < 2; ++again) {
    if (again) lq_tame_words<DT>(r);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = inf;
      hi[j] = -inf;
    }
#pragma unroll
    for (int t = 0; t < kLqPage; ++t) {
      float x[4];
      four(t, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = min_nan(lo[j], x[j]);
        hi[j] = max_nan(hi[j], x[j]);
      }
    }
    bool tame = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) tame = tame && lo[j] >= -65504.f && hi[j] <= 65504.f;  // (false for a NaN)
    if (__all_sync(0xffffffffu, tame)) break;
  }
  unsigned short* out = reinterpret_cast<unsigned short*>(codes) + lane;
  if (keys) {
    uint32_t w[4];
    float z[4], s[4], inv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = lq_group(lo[j], hi[j]);
      s[j] = half_lo(w[j]);
      z[j] = half_hi(w[j]);
      inv[j] = 1.0f / s[j];
    }
    *reinterpret_cast<uint4*>(meta + 16 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int t = 0; t < kLqPage; ++t) {
      float x[4];
      four(t, x);
      uint32_t c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c |= (uint32_t)lq_code(x[j], z[j], s[j], inv[j]) << (4 * j);
      st_code(out + 32 * t, c);
    }
  } else {
    const int j8 = lane & 7;
#pragma unroll
    for (int t0 = 0; t0 < kLqPage; t0 += 8) {
      float a[8], b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x[4];
        four(t0 + i, x);
        a[i] = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
        b[i] = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      }
#pragma unroll
      for (int o = 4, m = 4; o > 0; o >>= 1, m >>= 1) {  // m rows stay: those whose bit o is the lane's
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int i = 0; i < m; ++i) {
          const float ga = up ? a[i] : a[i + m], gb = up ? b[i] : b[i + m];
          const float ka = up ? a[i + m] : a[i], kb = up ? b[i + m] : b[i];
          a[i] = fminf(ka, __shfl_xor_sync(0xffffffffu, ga, o));
          b[i] = fmaxf(kb, __shfl_xor_sync(0xffffffffu, gb, o));
        }
      }
      const uint32_t own = lq_group(a[0], b[0]);
      const float own_inv = 1.0f / half_lo(own);
      *reinterpret_cast<uint32_t*>(meta + 16 * (t0 + j8) + 4 * (lane >> 3)) = own;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = __shfl_sync(0xffffffffu, own, (lane & 24) + i);
        const float inv = __shfl_sync(0xffffffffu, own_inv, (lane & 24) + i);
        const float s = half_lo(w), z = half_hi(w);
        float x[4];
        four(t0 + i, x);
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) c |= (uint32_t)lq_code(x[j], z, s, inv) << (4 * j);
        st_code(out + 32 * (t0 + i), c);
      }
    }
  }
}
#endif

}  // namespace mc
