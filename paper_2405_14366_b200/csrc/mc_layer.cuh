// Device pieces shared by the operators of an uncompressed layer's cache: what a query sees, what a score becomes.
#pragma once
#include "mc_common.cuh"

namespace mc {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// tanh(x) = x P(x^2) by reweighted least squares on tanh(x) / x: degree 4 on [-1/2, 1/2] (1.3e-8 relative), degree 6 on
// [-1, 1] (5e-8).
__host__ __device__ constexpr float tanh_tiny(int j) {
  return j == 0 ? 9.9999998687e-01f : j == 1 ? -3.3333069391e-01f : j == 2 ? 1.3324779261e-01f : j == 3 ? -5.2986071693e-02f : 1.7134999450e-02f;
}
__host__ __device__ constexpr float tanh_small(int j) {
  return j == 0   ? 9.9999995024e-01f
         : j == 1 ? -3.3332839133e-01f
         : j == 2 ? 1.3325203849e-01f
         : j == 3 ? -5.3457019959e-02f
         : j == 4 ? 2.0289962009e-02f
         : j == 5 ? -6.2033628195e-03f
                  : 1.0410172275e-03f;
}

// The score rule of a call (mc_score_opts) in the form the kernels use; scores are kept as log2(e) times their value,
// so that a probability is one instruction.
struct ScoreRule {
  const float* slopes;       // [n_q_heads] or null
  const int32_t* doc_start;  // [batch] or null
  const int32_t* prefix_len; // [batch] or null
  const int32_t* q_pos;      // [batch] or null
  float scale_log2;          // sm_scale * log2(e)
  float cap_inv;             // sm_scale / cap
  float cap_log2;            // cap * log2(e); 0: no cap
  int window;
};

static inline ScoreRule make_score_rule(const mc_score_opts* o) {
  ScoreRule r;
  r.slopes = o->alibi_slopes;
  r.doc_start = o->doc_start;
  r.prefix_len = o->prefix_len;
  r.q_pos = o->q_pos;
  r.scale_log2 = o->sm_scale * kLog2e;
  r.cap_inv = o->softcap > 0.f ? o->sm_scale / o->softcap : 0.f;
  r.cap_log2 = o->softcap > 0.f ? o->softcap * kLog2e : 0.f;
  r.window = o->window;
  return r;
}

#if defined(__CUDACC__)
// tanh to about 2 ulp.  |x| < 1.4: Lambert's continued fraction x / (1 + x^2 / (3 + x^2 / (5 + ...))) cut behind the
// 11, as one quotient (truncation below 1.7e-8 relative); larger: 1 - 2 / (1 + e^2x).  (__fdividef: 2 ulp, for denominators
// below 2^126; beyond, where e^2x is, it gives 0 and tanh is 1.)  The hardware's tanh
// instruction is good to 2^-11 only, which a cap of 50 would turn into an error of 0.02 in the exponent.
__device__ __forceinline__ float tanh_score(float x) {
  const float y = fabsf(x);
  if (y < 1.4f) {
    const float z = x * x;
    const float num = fmaf(z, fmaf(z, 21.f, 1260.f), 10395.f);
    const float den = fmaf(z, fmaf(z, z + 210.f, 4725.f), 10395.f);
    return x * __fdividef(num, den);
  }
  const float t = 1.f - __fdividef(2.f, 1.f + exp2f(fminf(y, 64.f) * (2.f * kLog2e)));
  return x != x ? x : copysignf(t, x);  // (fminf would turn a NaN into a number)
}
// 2^x to 2 ulp, one instruction: probabilities below 2^-126 are zero (exp2f's scaling of denormals costs as much again).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two binary32 numbers in one 64-bit register: sm_100's packed arithmetic does both in one issue slot.
__device__ __forceinline__ uint64_t pack2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// q . k -> score (log2 units), the cap included, the distance bias not.
__device__ __forceinline__ float score_of(const ScoreRule& r, float dot) {
  return r.cap_log2 > 0.f ? r.cap_log2 * tanh_score(dot * r.cap_inv) : dot * r.scale_log2;
}

// Four scores of a warp's lanes.  With a cap: x P(x^2) two at a time while every |x| of the warp is at most 1 (scores up
// to the cap itself before it), else the exact form.  The two differ in their last bits: what does not count comes as 0.
__device__ __forceinline__ void scores_of(const ScoreRule& r, float (&s)[4]) {
  if (!(r.cap_log2 > 0.f)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] *= r.scale_log2;
    return;
  }
  float big = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) big = fmaxf(big, fabsf(s[k] * r.cap_inv));
  if (__all_sync(0xffffffffu, big <= 1.f)) {
    const uint64_t inv = pack2(r.cap_inv, r.cap_inv), cap = pack2(r.cap_log2, r.cap_log2);
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const uint64_t x = mul2(pack2(s[k], s[k + 1]), inv), z = mul2(x, x);
      uint64_t q = pack2(tanh_small(6), tanh_small(6));
#pragma unroll
      for (int j = 5; j >= 0; --j) q = fma2(q, z, pack2(tanh_small(j), tanh_small(j)));
      unpack2(mul2(mul2(x, q), cap), s[k], s[k + 1]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = score_of(r, s[k]);
  }
}
// The largest of three numbers, and of one and two magnitudes (sm_100's three-input forms).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
  float r;
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// What one query sees: positions p with p <= q_pos and (p < prefix or p >= lo_pos).
struct View {
  int q_pos, prefix, lo_pos;
  __device__ __forceinline__ bool sees(int p) const { return p <= q_pos && (p < prefix || p >= lo_pos); }
};
__device__ __forceinline__ View view_at(const ScoreRule& r, int b, int q_pos) {
  View v;
  v.q_pos = q_pos;
  v.prefix = r.prefix_len ? r.prefix_len[b] : 0;
  v.lo_pos = r.doc_start ? r.doc_start[b] : 0;
  // (q_pos >= -1 and window >= 1: no overflow)
  if (r.window > 0) v.lo_pos = max(v.lo_pos, q_pos - r.window + 1);
  return v;
}
#endif

}  // namespace mc
