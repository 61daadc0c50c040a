// Products of few tokens' codes with stored 8-bit weights (Sec. 4.1's deployed setting: per-token activations,
// per-channel symmetric weights):  Y[t,o] = step_t * step_o * sum_c code[t,c] * wcode[o,c].
// More tokens take the tiles of gemm_i8.hip.
#include "contraction.h"

namespace tlq {

// A block computes 16 outputs for 16 NT tokens; its waves split the row of codes and meet in LDS (integer sums: exact, in
// any order).  16x16x64 MFMA with the weights as rows: a lane holds 16 codes of output lane % 16, which it reads from
// memory as they are, 64 consecutive bytes a row and instruction; nothing passes through LDS before the sums.
// Bound by the bytes of the weights: every one is read once per 16 NT tokens.
template <int NT, int NW>
__global__ __launch_bounds__(NW * 64) void linear_few_kernel(LinearI8Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(16))) i32x4 red[NW][NT][64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t o0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * (16 * NT);
  const int chunks = (int)(a.K >> 6);                   // of 64 codes
  const int c0 = (int)((int64_t)chunks * wave / NW), c1 = (int)((int64_t)chunks * (wave + 1) / NW);
  const int64_t o = o0 + l16 < a.c_out ? o0 + l16 : a.c_out - 1;
  const int8_t* w = a.wc + o * a.ldw + fq * 16;
  const int8_t* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = t0 + n * 16 + l16 < a.n_tok ? t0 + n * 16 + l16 : a.n_tok - 1;
    x[n] = a.xc + t * a.ldx + fq * 16;
  }
  i32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = i32x4{0, 0, 0, 0};
  constexpr int U = NT == 1 ? 8 : 4;
  int c = c0;
  auto some = [&](auto count) {
    constexpr int N = decltype(count)::value;
    i32x4 wv[N], xv[N][NT];
#pragma unroll
    for (int u = 0; u < N; ++u) wv[u] = *reinterpret_cast<const i32x4*>(w + (int64_t)(c + u) * 64);
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) xv[u][n] = *reinterpret_cast<const i32x4*>(x[n] + (int64_t)(c + u) * 64);
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], xv[u][n], acc[n], 0, 0, 0);
    c += N;
  };
  while (c + U <= c1) some(std::integral_constant<int, U>{});
  while (c < c1) some(std::integral_constant<int, 1>{});
#pragma unroll
  for (int n = 0; n < NT; ++n) red[wave][n][lane] = acc[n];
  __syncthreads();
  if (wave >= NT) return;
  i32x4 s = red[0][wave][lane];
#pragma unroll
  for (int v = 1; v < NW; ++v) s += red[v][wave][lane];
  const int64_t t = t0 + wave * 16 + l16, oq = o0 + fq * 4;
  if (t >= a.n_tok) return;
  const float st = a.xs[t];
  float y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = oq + r < a.c_out ? st * (a.ws[oq + r] * (float)s[r]) : 0.0f;
  if (oq + 3 < a.c_out) store_y4(a.Y, a.ydt, t * a.ldy + oq, y);
  else
    for (int r = 0; r < 3; ++r)
      if (oq + r < a.c_out) store_y1(a.Y, a.ydt, t * a.ldy + oq + r, y[r]);
#endif
}

hipError_t launch_linear_few(const LinearI8Args& a, hipStream_t stream) {
  ProfScope ps("linear_few", stream, (double)a.c_out * (double)a.K);
  const unsigned bo = (unsigned)ceil_div(a.c_out, 16);
  auto go = [&](auto kern, int waves, int tokens) { kern<<<dim3(bo, (unsigned)ceil_div(a.n_tok, tokens)), waves * 64, 0, stream>>>(a); };
  if (a.n_tok <= 16) go(linear_few_kernel<1, 16>, 16, 16);
  else if (a.n_tok <= 32) go(linear_few_kernel<2, 16>, 16, 32);
  else if (a.n_tok <= 48) go(linear_few_kernel<3, 16>, 16, 48);
  else go(linear_few_kernel<4, 16>, 16, 64);
  return hipGetLastError();
}

}  // namespace tlq
