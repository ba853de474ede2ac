// Device pieces shared by the operators of an uncompressed layer's cache: what a query sees, what a score becomes.
#pragma once
#include "mc_common.cuh"

namespace mc {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// The score rule of a call (mc_score_opts) in the form the kernels use; scores are kept as log2(e) times their value,
// so that a probability is one exp2f.
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
// 11, as one quotient (truncation below 1.7e-8 relative); larger: 1 - 2 / (1 + e^2x).  The hardware's tanh
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
// q . k -> score (log2 units), the cap included, the distance bias not.
__device__ __forceinline__ float score_of(const ScoreRule& r, float dot) {
  return r.cap_log2 > 0.f ? r.cap_log2 * tanh_score(dot * r.cap_inv) : dot * r.scale_log2;
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
