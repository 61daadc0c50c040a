// What stands between two products of a block in 8 bits: the residual's addition, the root-mean-square norm and the codes of the
// normalised rows, in one pass over the residual stream.
//
// This file is compiled with floating-point contraction off: every float operation below rounds exactly once, in the order
// written, so the codes and steps are reproducible bit for bit.
#include "quant_codes.h"

namespace tlq {

struct NormCodesDev {
  const uint16_t *H, *Z; int64_t ldh, ldz, n, c;
  const float* w; float eps, qa;
  uint16_t* out; int64_t ldo;
  int8_t* codes; int64_t ldc; float* steps;
};

// h = round16(H + Z); u = (h * r) * w with r = 1 / sqrt(mean h^2 + eps); code = rint(u / step), step = max |u| / qa.
// W waves have a row, P passes of 512 W channels, which stay in registers from the sum through the maximum to the codes, so that
// H and Z are read once.  The squares of 16-bit numbers are exact in double and their sum is off by 2^-46 of itself at
// most (85 additions one behind the other for 65,536 channels), so that r is the float that the definition gives, but where 1 / sqrt lies
// that near between two (a row in some millions).  With one wave a row
// a block has four rows.  Bound by bytes: 10,240 x 5120 with the residual 77 us, 4.8 TB/s of seven bytes an element (a copy reaches
// 4.8), x 4096 60, x 8192 112, 4000 x 13824 86, 2000 x 32,768 107; by latency for few rows, 1 x 4096 3.6.  Beyond 32,768 channels
// the eight passes do not all fit into the 128 registers of a block of 16 waves, 30 are kept in scratch: 2000 x 32,776 206 us, x
// 40,000 233 (2.4 TB/s), x 65,536 322 (2.8 TB/s).
template <typename T, int W, int P>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void add_norm_codes_kernel(NormCodesDev a) {
  __shared__ double sums[W];
  __shared__ float tops[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (W == 1 && row >= a.n) return;
  const int c0 = ((W == 1 ? 0 : wave) * 64 + lane) * 8;
  uint4 h[P];
  double sum = 0.0;
  constexpr int B = P < 4 ? P : 4;      // passes whose loads are issued at once
#pragma unroll
  for (int p0 = 0; p0 < P; p0 += B) {
    uint4 z[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int64_t c = c0 + (p0 + i) * (512 * W);
      h[p0 + i] = c < a.c ? *reinterpret_cast<const uint4*>(a.H + row * a.ldh + c) : make_uint4(0, 0, 0, 0);
      if (a.Z) z[i] = c < a.c ? *reinterpret_cast<const uint4*>(a.Z + row * a.ldz + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int64_t c = c0 + (p0 + i) * (512 * W);
      float x[8];
      widen8<T>(h[p0 + i], x);
      if (a.Z) {
        float y[8];
        widen8<T>(z[i], y);
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint16_t lo = T::from_float(x[2 * j] + y[2 * j]), hi = T::from_float(x[2 * j + 1] + y[2 * j + 1]);
          x[2 * j] = T::to_float(lo);
          x[2 * j + 1] = T::to_float(hi);
          o[j] = (uint32_t)lo | (uint32_t)hi << 16;
        }
        h[p0 + i] = make_uint4(o[0], o[1], o[2], o[3]);
      }
      if (a.out && c < a.c) *reinterpret_cast<uint4*>(a.out + row * a.ldo + c) = h[p0 + i];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)x[j], (double)x[j], sum);
    }
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
  if constexpr (W > 1) {
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = sums[0];
#pragma unroll
    for (int i = 1; i < W; ++i) sum += sums[i];
  }
  const float r = (float)(1.0 / sqrt(sum / (double)a.c + (double)a.eps));
  float m = 0.0f;
  float u[8], f[8];
  auto normed = [&](int p) {       // (behind c zeros, whatever the weights are)
    const int64_t c = c0 + p * (512 * W);
    float x[8];
    widen8<T>(h[p], x);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 1.0f;
    if (a.w && c < a.c) load8(a.w + c, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = (x[j] * r) * f[j];
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    normed(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(u[j]));
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if constexpr (W > 1) {
    if (lane == 0) tops[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, tops[i]);
  }
  Grid g;
  g.delta = fmaxf(m, kRangeFloor) / a.qa;
  g.rd = __builtin_amdgcn_rcpf(g.delta);
  g.lim = g.delta < 1e36f ? 0.49999976f - 4.8e-7f * (a.qa + 1.0f) : -1.0f;
  // (a row that is not finite has a mean that is not, and r of zero or NaN; a mean of zero an infinite r)
  if (lane == 0 && (W == 1 || wave == 0)) a.steps[row] = r > 0.0f && r < INFINITY ? g.delta : NAN;
  const int64_t end = (a.c + 127) / 128 * 128;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t c = c0 + p * (512 * W);
    if (c >= end) break;
    normed(p);
    float q[8];
    if (!(rint_quotient8(u, g, 0.0f, q) < g.lim)) divide8(u, g, q);
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = __builtin_amdgcn_fmed3f(q[j], -a.qa - 1.0f, a.qa);
    *reinterpret_cast<uint2*>(a.codes + row * a.ldc + c) = make_uint2(pack_i8(q[0], q[1], q[2], q[3]), pack_i8(q[4], q[5], q[6], q[7]));
  }
}

hipError_t launch_add_norm_codes(const void* H, int64_t ldh, const void* Z, int64_t ldz, int64_t n, int64_t c, const float* w, float eps,
                                 int bits, bool bf16, void* out, int64_t ldo, int8_t* codes, int64_t ldc, float* steps, hipStream_t stream) {
  ProfScope ps("add_norm_codes", stream, (Z ? 7.0 : 3.0) * (double)n * (double)c);
  const NormCodesDev a{(const uint16_t*)H, (const uint16_t*)Z, ldh, ldz, n, c, w, eps, (float)((1 << (bits - 1)) - 1),
                       (uint16_t*)out, ldo, codes, ldc, steps};
  auto go = [&](auto kern, int waves) {
    kern<<<(unsigned)(waves == 1 ? ceil_div(n, 4) : n), (waves == 1 ? 256 : waves * 64), 0, stream>>>(a);
  };
  auto pick = [&](auto t) {
    using T = decltype(t);
    if (c <= 1024) go(add_norm_codes_kernel<T, 1, 2>, 1);
    else if (c <= 4096) go(add_norm_codes_kernel<T, 4, 2>, 4);
    else if (c <= 8192) go(add_norm_codes_kernel<T, 4, 4>, 4);
    else if (c <= 16384) go(add_norm_codes_kernel<T, 8, 4>, 8);
    else if (c <= 32768) go(add_norm_codes_kernel<T, 16, 4>, 16);
    else go(add_norm_codes_kernel<T, 16, 8>, 16);
  };
  bf16 ? pick(BF16{}) : pick(F16{});
  return hipGetLastError();
}

}  // namespace tlq
