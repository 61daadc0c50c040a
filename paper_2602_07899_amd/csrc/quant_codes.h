// What the kernels that make signed codes share.  For files that are compiled with floating-point contraction off: every float
// operation rounds exactly once, in the order written.
#pragma once
#include "common.h"

namespace tlq {

// Grid of one group: step, an approximate reciprocal, zero point, and how near to a tie the reciprocal may be used.
struct Grid { float delta, rd, zpf, lim; };

// The integer codes need rint(fl(x / delta)).  With rd within one ulp of 1/delta, t = fl(x * rd) lies
// within 2.4e-7 |t| of the rounded quotient, so rint(t) is that integer unless a half-integer sits inside
// the gap; |t - rint(t)| < lim = 0.49999976 - 4.8e-7 max|t| rules that out for a whole group (with a factor of two to
// spare), and the rare rest (one element in 10^5 at 4 bits) is divided, eight elements at a time.
// Outside [1e-5, 1e36) and for NaN lim is negative or NaN: everything is divided.
// rint(fl(ws / delta)) of eight values unless the result, or `tie` from before, reaches lim; the larger of the two measures
__device__ __forceinline__ float rint_quotient8(const float (&ws)[8], const Grid& g, float tie, float (&n)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float t = ws[j] * g.rd;
    n[j] = rintf(t);
    tie = fmaxf(tie, fabsf(t - n[j]));
  }
  return tie;
}
__device__ __forceinline__ void divide8(const float (&ws)[8], const Grid& g, float (&n)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    n[j] = rintf(ws[j] / g.delta);
    asm volatile("" : "+v"(n[j]) :: "memory");     // one after the other, and in a branch, not computed and dropped
  }
}

__device__ __forceinline__ void load8(const float* __restrict__ p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void widen8(const uint4& v, float (&w)[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = T::to_float((uint16_t)(u[j >> 1] >> ((j & 1) * 16)));
}
__device__ __forceinline__ void times8(const float (&w)[8], const float (&s)[8], float (&ws)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) ws[j] = w[j] * s[j];
}
// four small integers as bytes: beside 1.5 * 2^23 the low byte of the float is the integer's
__device__ __forceinline__ uint32_t pack_i8(float a, float b, float c, float d) {
  auto bits = [](float v) { return __builtin_bit_cast(uint32_t, v + 12582912.0f); };
  return __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400u) | __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0cu);
}

}  // namespace tlq
