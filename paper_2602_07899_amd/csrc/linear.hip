// Products of few tokens' codes with stored 8-bit weights (Sec. 4.1's deployed setting: per-token activations,
// per-channel symmetric weights):  Y[t,o] = step_t * step_o * sum_c code[t,c] * wcode[o,c].
// More tokens take the tiles of gemm_i8.hip.
#include "contraction.h"

namespace tlq {

#if defined(__HIP_DEVICE_COMPILE__)
// four neighbouring outputs of a token
__device__ __forceinline__ void write4(const LinearI8Args& a, int64_t t, int64_t o, float st, const i32x4& s) {
  float y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = o + r < a.c_out ? st * (a.ws[o + r] * (float)s[r]) : 0.0f;
  if (o + 3 < a.c_out) store_y4(a.Y, a.ydt, t * a.ldy + o, y);
  else
    for (int r = 0; r < 3; ++r)
      if (o + r < a.c_out) store_y1(a.Y, a.ydt, t * a.ldy + o + r, y[r]);
}
#endif

// A block computes 16 outputs for 16 NT tokens; its waves split the row of codes and meet in LDS (integer sums: exact, in
// any order).  16x16x64 MFMA with the weights as rows: a lane holds 16 codes of output lane % 16 (32 neighbouring ones in two
// products, so that four lanes read a whole line), which it reads from memory as they are; nothing passes through LDS
// before the sums.
// Bound by the bytes of the weights, every one is read once per 16 NT tokens, and by latency where they are few: 1 x 4096 x 4096
// 5.4 us, 3.1 TB/s.
template <int NT, int NW>
__global__ __launch_bounds__(NW * 64) void linear_few_kernel(LinearI8Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(16))) i32x4 red[NW][NT][64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t o0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * (16 * NT);
  const int chunks = (int)(a.K >> 7);                   // of 128 codes: two products
  const int c0 = (int)((int64_t)chunks * wave / NW), c1 = (int)((int64_t)chunks * (wave + 1) / NW);
  const int64_t o = o0 + l16 < a.c_out ? o0 + l16 : a.c_out - 1;
  const int8_t* w = a.wc + o * a.ldw + fq * 32;
  const int8_t* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = t0 + n * 16 + l16 < a.n_tok ? t0 + n * 16 + l16 : a.n_tok - 1;
    x[n] = a.xc + t * a.ldx + fq * 32;
  }
  i32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = i32x4{0, 0, 0, 0};
  constexpr int U = NT == 1 ? 4 : 2;
  int c = c0;
  auto some = [&](auto count) {
    constexpr int N = 2 * decltype(count)::value;
    i32x4 wv[N], xv[N][NT];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int at = (c + u / 2) * 128 + u % 2 * 16;
      wv[u] = *reinterpret_cast<const i32x4*>(w + at);
#pragma unroll
      for (int n = 0; n < NT; ++n) xv[u][n] = *reinterpret_cast<const i32x4*>(x[n] + at);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], xv[u][n], acc[n], 0, 0, 0);
    c += N / 2;
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
  const int64_t t = t0 + wave * 16 + l16;
  if (t < a.n_tok) write4(a, t, o0 + fq * 4, a.xs[t], s);
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

// More tokens: 128 outputs x 16 NT tokens a block, one of `splits` parts of the row of codes.  The tokens' codes are shared by
// the block's waves through LDS (512 codes a stage, two stages); the weights are read once and by one wave each, so they go from
// memory to registers, 512 codes ahead.  Waves 0 - 3 and 4 - 7 have the same four groups of 32 outputs and every second 128
// codes.  Sums of one part are whole numbers; with several parts they go to the workspace and linear_join_kernel adds them.
// Reading the tokens' codes from memory in every wave, as above, costs as much as the weights for each 16 tokens (see
// linear_kind for both sides).  48 x 11008 x 4096 13.9 us, 3.2 TB/s of weights (weights that are in the caches take 13: two and
// a half stages a block, so the first loads and the meeting count), and 4.0 for the sums of eight parts.  Weights two stages
// ahead instead of one: calls of 48 x 11008 x 4096 23.1 25.4, 64 x 4096 x 11008 24.3 26.6.
constexpr int kMidStage = 512;
template <int NT>
__global__ __launch_bounds__(512) void linear_mid_kernel(LinearI8Args a, int splits, int* __restrict__ partial) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int ROWS = 16 * NT, PER = ROWS * kMidStage / 16 / 512;      // 16-byte pieces of a stage for a thread
  static_assert(PER >= 1, "stage");
  __shared__ __attribute__((aligned(1024))) int8_t lds[2][ROWS * kMidStage];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int og = wave & 3, kh = wave >> 2;
  const int64_t o0 = (int64_t)blockIdx.x * 128 + og * 32, t0 = (int64_t)blockIdx.y * ROWS;
  const int part = blockIdx.z, chunks = (int)(a.K >> 7);      // of 128 codes
  const int c0 = (int)((int64_t)chunks * part / splits), c1 = (int)((int64_t)chunks * (part + 1) / splits);
  const int8_t* w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t o = o0 + i * 16 + l16 < a.c_out ? o0 + i * 16 + l16 : a.c_out - 1;
    w[i] = a.wc + o * a.ldw + fq * 32;
  }
  // a row of a stage: 32 pieces of 16 codes, piece p at p ^ row % 16 (the lanes of a fragment read name 16 rows)
  const int8_t* xp[PER];
  int at[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int row = (i * 512 + tid) >> 5, piece = tid & 31;
    const int64_t t = t0 + row < a.n_tok ? t0 + row : a.n_tok - 1;
    xp[i] = a.xc + t * a.ldx + piece * 16;
    at[i] = row * kMidStage + ((piece ^ (row & 15)) << 4);
  }
  const int piece = tid & 31;
  i32x4 xr[PER], wr[2][4], acc[2][NT];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[i][n] = i32x4{0, 0, 0, 0};
  // (pieces and weights behind the part's end: the row's last ones stand in, their products are not taken)
  auto load_x = [&](int c) {
    const int over = c + (piece >> 3) - (c1 - 1);
    const int off = (c - (over > 0 ? over : 0)) * 128;
#pragma unroll
    for (int i = 0; i < PER; ++i) xr[i] = *reinterpret_cast<const i32x4*>(xp[i] + off);
  };
  auto load_w = [&](int c, int g) {      // the wave's g-th 128 codes of the stage that begins at c
    const int k = c + 2 * g + kh < c1 ? c + 2 * g + kh : c1 - 1;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) wr[g][i * 2 + u] = *reinterpret_cast<const i32x4*>(w[i] + k * 128 + u * 16);
  };
  auto store_x = [&](int8_t* to) {
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<i32x4*>(to + at[i]) = xr[i];
  };
  load_x(c0);
  load_w(c0, 0);
  load_w(c0, 1);
  store_x(lds[0]);
  int cur = 0;
  for (int c = c0; c < c1; c += 4, cur ^= 1) {
    __syncthreads();
    const bool more = c + 4 < c1;
    if (more) load_x(c + 4);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if (c + 2 * g + kh < c1) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const i32x4 x = *reinterpret_cast<const i32x4*>(lds[cur] + (n * 16 + l16) * kMidStage +
                                                            (((2 * g + kh) * 8 + fq * 2 + u ^ l16) << 4));
            acc[0][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[g][u], x, acc[0][n], 0, 0, 0);
            acc[1][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[g][2 + u], x, acc[1][n], 0, 0, 0);
          }
      }
      if (more) load_w(c + 4, g);
    }
    if (more) store_x(lds[cur ^ 1]);
  }
  // the two halves of the codes meet in LDS
  __syncthreads();
  i32x4* meet = reinterpret_cast<i32x4*>(&lds[0][0]);      // [group of outputs][2 NT][64]
  if (kh) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) meet[(og * 2 * NT + i * NT + n) * 64 + lane] = acc[i][n];
  }
  __syncthreads();
  if (kh) return;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = t0 + n * 16 + l16;
    if (t >= a.n_tok) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const i32x4 s = acc[i][n] + meet[(og * 2 * NT + i * NT + n) * 64 + lane];
      const int64_t o = o0 + i * 16 + fq * 4;
      if (splits > 1) {      // (rows of whole fours)
        if (o < a.c_out) *reinterpret_cast<i32x4*>(partial + ((int64_t)part * a.n_tok + t) * ((a.c_out + 3) & ~(int64_t)3) + o) = s;
        continue;
      }
      write4(a, t, o, a.xs[t], s);
    }
  }
#endif
}

__global__ __launch_bounds__(256) void linear_join_kernel(LinearI8Args a, int splits, const int* __restrict__ partial) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int64_t quads = (a.c_out + 3) >> 2, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n_tok * quads) return;
  const int64_t t = i / quads;
  i32x4 s = *reinterpret_cast<const i32x4*>(partial + i * 4);
#pragma unroll 8
  for (int p = 1; p < splits; ++p) s += *reinterpret_cast<const i32x4*>(partial + ((int64_t)p * a.n_tok * quads + i) * 4);
  write4(a, t, (i - t * quads) * 4, a.xs[t], s);
#endif
}

// Which kernels are the fastest, by whole calls (the token's codes among them; a graph of calls, weights that change from
// call to call), us few, shared tokens, tiles of the search:
//   n x channels x outputs
//   16 x 4096 x 4096    10.3 14.2 21.5     64 x 4096 x 4096   16.0 18.5 23.9     128 x 4096 x 4096    -  19.8 22.8
//   16 x 11008 x 4096   20.0 21.3 46.1     48 x 11008 x 4096  29.4 23.5 50.7     128 x 11008 x 4096   -  30.1 60.5
//   16 x 5120 x 13824   30.5 26.5 31.6     64 x 11008 x 4096  34.6 24.9 54.4     128 x 4096 x 11008   -  32.4 28.3
//   32 x 4096 x 4096    12.0 15.3 22.1     64 x 4096 x 11008  39.0 23.6 26.8     256 x 4096 x 4096    -  24.9 24.1
//   32 x 4096 x 11008   26.0 21.4 24.9     64 x 5120 x 13824  64.1 30.7 38.3     256 x 11008 x 4096   -  43.4 58.6
//   16 x 1096 x 1399     6.2 10.0 11.2     300 x 1096 x 1399  12.5 15.1 15.1     256 x 4096 x 11008   -  48.0 29.5
// Up to 64 tokens the few kernel's bytes decide, the weights once for each 16 tokens; beyond, whether its blocks run in one round
// and are short, then whether the tiles of 128 x 128 are so few that most CUs have none, and their contraction long.  Few
// and the better of the others: 128 x 1096 x 1399 8.3 14.8, 128 x 2048 x 2048 10.7 14.5, 300 x 1096 x 1399 12.5 15.0, 300 x 2048 x
// 1399 16.7 19.1, 1000 x 128 x 500 8.7 10.3, 400 x 1096 x 1000 13.2 14.2, 128 x 2048 x 4096 (512 blocks) 16.8 16.9, 4000 x 2048 x 128
// (504) 25.2 23.2, 613 x 1096 x 1399 (880) 21.4 15.8, 96 x 3000 x 4000 19.9 18.4, 100 x 8192 x 1024 25.4 19.7.
// (Codes and product of up to four tokens in one launch, every block making the codes for itself: 1 x 4096 x 4096 9.0 -> 12.9,
// 1 x 11008 x 4096 16.1 -> 18.6.)
LinearKind linear_kind(int64_t n_tok, int64_t c_out, int64_t K) {
  if (n_tok <= 64) return (double)ceil_div(n_tok, 16) * (double)c_out * (double)K <= 70e6 ? kLinearFew : kLinearMid;
  if (K <= 2048 && ceil_div(n_tok, 64) * ceil_div(c_out, 16) <= 448) return kLinearFew;
  return n_tok <= kLinearMidTokens && ceil_div(n_tok, 128) * ceil_div(c_out, 128) <= 64 && K >= 2048 ? kLinearMid : kLinearTiles;
}

int linear_mid_splits(int64_t n_tok, int64_t c_out, int64_t K) {
  const int64_t blocks = ceil_div(c_out, 128) * ceil_div(n_tok, 64), most = ceil_div(K, kMidStage);
  int64_t s = 256 / blocks;
  if (s > most) s = most;
  if (s > 16) s = 16;
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_linear_mid(const LinearI8Args& a, int splits, int* partial, hipStream_t stream) {
  {
    ProfScope ps("linear_mid", stream, (double)a.c_out * (double)a.K);
    auto go = [&](auto kern, int tokens) {
      kern<<<dim3((unsigned)ceil_div(a.c_out, 128), (unsigned)ceil_div(a.n_tok, tokens), (unsigned)splits), 512, 0, stream>>>(a, splits, partial);
    };
    if (a.n_tok <= 16) go(linear_mid_kernel<1>, 16);
    else if (a.n_tok <= 32) go(linear_mid_kernel<2>, 32);
    else if (a.n_tok <= 48) go(linear_mid_kernel<3>, 48);
    else go(linear_mid_kernel<4>, 64);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess || splits == 1) return e;
  ProfScope ps("linear_join", stream, 4.0 * splits * (double)a.n_tok * (double)a.c_out);
  linear_join_kernel<<<(unsigned)ceil_div(a.n_tok * ((a.c_out + 3) >> 2), 256), 256, 0, stream>>>(a, splits, partial);
  return hipGetLastError();
}

}  // namespace tlq
