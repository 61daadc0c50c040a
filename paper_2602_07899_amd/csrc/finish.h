// The epilogue of a product: bias, activation, and a second matrix that is added or multiplied.
#pragma once
#include "common.h"

namespace tlq {

enum { kActNone = 0, kActGate = 1, kActErf = 2 };      // v; v times a logistic function; v times the normal distribution
inline int act_class(int act) { return act == TLQ_ACT_NONE ? kActNone : act == TLQ_ACT_GELU_ERF ? kActErf : kActGate; }

#if defined(__HIP_DEVICE_COMPILE__)
// v / (1 + exp(-(c1 v + c3 v^3))): SiLU with 1 and 0; GELU in its tanh form with 2 sqrt(2/pi) and 0.044715 times that, since
// (1 + tanh(x)) / 2 = 1 / (1 + exp(-2 x)).  k1, k3 are these times -log2(e).  The roundings of the exponent come to 4 |x| 2^-24 of
// a result in the tail, about what those of v itself do there.  (v is held to 2^60 in the exponent, where 0 v^3 is to be 0.)
__device__ __forceinline__ float act_gate(float v, float k1, float k3) {
  const float m = __builtin_amdgcn_fmed3f(v, -0x1p60f, 0x1p60f);
  return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(m * __builtin_fmaf(k3 * m, m, k1)));
}
// v Phi(v) = v - v erfc(v / sqrt 2) / 2 for v >= 0, -|v| erfc(|v| / sqrt 2) / 2 below, which keeps its relative precision where
// 1 + erf cancels.  erfc(z) exp(z^2) = s P(s), s = 1 / (1 + z / 2), with P of degree 8 fitted here to the least relative
// error on 0 <= z <= 10 (1.7e-7 as floats); beyond, exp(-z^2) is no float, and |v| is held to 30 so that nothing times infinity
// stands there.
__device__ __forceinline__ float act_erf(float v) {
  const float m = __builtin_amdgcn_fmed3f(v, -30.0f, 30.0f);
  const float z = fabsf(m) * 0.707106769f, s = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.5f, 1.0f));
  float q = -0.0590690114f;
  q = __builtin_fmaf(q, s, 0.284575194f);
  q = __builtin_fmaf(q, s, -0.48720035f);
  q = __builtin_fmaf(q, s, 0.278067678f);
  q = __builtin_fmaf(q, s, -0.0266259946f);
  q = __builtin_fmaf(q, s, 0.202686995f);
  q = __builtin_fmaf(q, s, 0.243103728f);
  q = __builtin_fmaf(q, s, 0.282375306f);
  q = __builtin_fmaf(q, s, 0.282086432f);
  const float tail = 0.5f * m * (s * q) * __builtin_amdgcn_exp2f(m * (m * -0.721347520f));      // v erfc(|v| / sqrt 2) / 2
  return v < 0.0f ? tail : v - tail;      // (NaN stays)
}
template <int CLASS>
__device__ __forceinline__ float act_of(float v, const Finish& f) {
  if constexpr (CLASS == kActNone) return v;
  else if constexpr (CLASS == kActErf) return act_erf(v);
  else return act_gate(v, f.k1, f.k3);
}
// by the call's activation, the same for a whole launch
__device__ __forceinline__ float act_of(float v, const Finish& f) {
  if (f.act == TLQ_ACT_NONE) return v;
  return f.act == TLQ_ACT_GELU_ERF ? act_erf(v) : act_gate(v, f.k1, f.k3);
}
#endif

}  // namespace tlq
