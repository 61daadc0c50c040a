// The epilogue of a product: bias, activation, and a second matrix that is added or multiplied.
#pragma once
#include "common.h"

namespace tlq {

enum { kActNone = 0, kActGate = 1, kActErf = 2 };      // v; v times a logistic function; v times the normal distribution
inline int act_class(int act) { return act == TLQ_ACT_NONE ? kActNone : act == TLQ_ACT_GELU_ERF ? kActErf : kActGate; }

#if defined(__HIP_DEVICE_COMPILE__)
// exp(-x), x = hi + lo: the product with log2(e) in two parts, since what its rounding loses is a multiple of |x| ulps of the result
__device__ __forceinline__ float exp_minus(float hi, float lo) {
  constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f;      // (together log2(e) to 2^-50)
  const float t = -hi * kLog2e;
  const float rest = __builtin_fmaf(-hi, kLog2e, -t) - __builtin_fmaf(hi, kLog2eLow, lo * kLog2e);
  const float e = __builtin_amdgcn_exp2f(t);
  return e * __builtin_fmaf(rest, 0.693147182f, 1.0f);
}
// v / (1 + exp(-(k1 v + k3 v^3))): SiLU with 1 and 0; GELU in its tanh form with 2 sqrt(2/pi) and 0.044715 times that, since
// (1 + tanh(x)) / 2 = 1 / (1 + exp(-2 x)).  (Held where the exponential is zero or no float: the product of an infinity's parts
// would be NaN.)
__device__ __forceinline__ float act_gate(float v, float k1, float k3) {
  const float x = v * __builtin_fmaf(k3 * v, v, k1);
  return v * __builtin_amdgcn_rcpf(1.0f + exp_minus(__builtin_amdgcn_fmed3f(x, -1000.0f, 1000.0f), 0.0f));
}
// v Phi(v) = v - v erfc(v / sqrt 2) / 2 for v >= 0, -|v| erfc(|v| / sqrt 2) / 2 below, which keeps its relative precision where
// 1 + erf cancels.  erfc(z) exp(z^2) = s P(s), s = 1 / (1 + z / 2), with P of degree 8 fitted here to the least relative
// error on 0 <= z <= 10 (1.7e-7 as floats); beyond, exp(-z^2) is no float.
__device__ __forceinline__ float act_erf(float v) {
  const float z = fabsf(v) * 0.707106769f, s = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.5f, 1.0f));
  float q = -0.0590690114f;
  q = __builtin_fmaf(q, s, 0.284575194f);
  q = __builtin_fmaf(q, s, -0.48720035f);
  q = __builtin_fmaf(q, s, 0.278067678f);
  q = __builtin_fmaf(q, s, -0.0266259946f);
  q = __builtin_fmaf(q, s, 0.202686995f);
  q = __builtin_fmaf(q, s, 0.243103728f);
  q = __builtin_fmaf(q, s, 0.282375306f);
  q = __builtin_fmaf(q, s, 0.282086432f);
  const float half = 0.5f * v, hi = fminf(half * v, 100.0f), lo = hi < 100.0f ? __builtin_fmaf(half, v, -hi) : 0.0f;      // v^2 / 2 in two parts
  const float tail = half * (s * q) * exp_minus(hi, lo);      // v erfc(|v| / sqrt 2) / 2
  return v >= 0.0f ? v - tail : tail;
}
__device__ __forceinline__ float act_of(float v, const Finish& f) {
  if (f.act == TLQ_ACT_NONE) return v;
  if (f.act == TLQ_ACT_GELU_ERF) return act_erf(v);
  return act_gate(v, f.k1, f.k3);
}
template <int CLASS>
__device__ __forceinline__ float act_of(float v, const Finish& f) {
  if constexpr (CLASS == kActNone) return v;
  else if constexpr (CLASS == kActErf) return act_erf(v);
  else return act_gate(v, f.k1, f.k3);
}
#endif

}  // namespace tlq
