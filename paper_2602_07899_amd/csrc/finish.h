// The epilogue of a product: bias, activation, and a second matrix that is added or multiplied.
#pragma once
#include "common.h"

namespace tlq {

enum { kActNone = TLQ_ACT_NONE, kActSilu = TLQ_ACT_SILU, kActTanh = TLQ_ACT_GELU_TANH, kActErf = TLQ_ACT_GELU_ERF };

#if defined(__HIP_DEVICE_COMPILE__)
// v / (1 + exp(-v)), the exponent in powers of two
__device__ __forceinline__ float act_silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));
}
// The same of c1 v + c3 v^3, c1 = 2 sqrt(2/pi), c3 = 0.044715 c1, since (1 + tanh(x)) / 2 = 1 / (1 + exp(-2 x)).  The roundings of the
// exponent come to 4 |x| 2^-24 of a result in the tail, about what those of v itself do there.
__device__ __forceinline__ float act_tanh(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * __builtin_fmaf(-0.102943240f * v, v, -2.30220820f)));
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
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
  if constexpr (ACT == kActNone) return v;
  else if constexpr (ACT == kActSilu) return act_silu(v);
  else if constexpr (ACT == kActTanh) return act_tanh(v);
  else return act_erf(v);
}
// by the call's activation, the same for a whole launch
__device__ __forceinline__ float act_of(float v, int act) {
  if (act == kActNone) return v;
  return act == kActSilu ? act_silu(v) : act == kActTanh ? act_tanh(v) : act_erf(v);
}
#endif

}  // namespace tlq
