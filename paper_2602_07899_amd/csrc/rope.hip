// Queries and keys of a decoder block: normalised for each head and rotated by their position, in one pass.
#include <type_traits>

#include "common.h"

namespace tlq {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

// u = x / sqrt(mean x^2 + eps) * w over the head_dim channels of a head, then the pair (u_a, u_b) turned by
// pos * inv_freq[i].  DH / 8 lanes hold a head, eight channels each, so a wave has 512 / DH heads of one token at a time.
// The angles belong to the token: a wave computes each cosine and sine once (a lane one or two of them, through LDS) and
// uses them for all heads it takes.  Angles are reduced to a fraction of a turn in double: at position 2^31 a float
// product would be off by whole turns.
// Bound by the bytes of Q and K, read and written once.
template <typename T, int DH, bool PAIRS, bool NORM, bool NT>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkRopeArgs a, int wpt, bool nts) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPH = DH / 8, HPW = 64 / LPH;
  __shared__ __attribute__((aligned(16))) float cs[4][2][DH / 2];
  const int lane = threadIdx.x & 63, sub = lane & (LPH - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = (int64_t)blockIdx.x * (4 / wpt) + wave / wpt;
  if (t >= a.n_tok) return;                       // (no barrier below)
  const int half = a.rot >> 1;
  {
    const double p = (double)a.pos[t];
    for (int i = lane; i < half; i += 64) {
      double turns = p * a.inv_freq[i] * 0.15915494309189535;
      turns -= __builtin_rint(turns);
      float s, c;
      sincospif(2.0f * (float)turns, &s, &c);
      cs[wave][0][i] = c;
      cs[wave][1][i] = s;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  // this lane's channels: pairs of neighbours, or the lower or upper half of pairs rot / 2 apart
  const int d0 = sub * 8, hs = half >> 3;         // (rot is a multiple of 16)
  const bool turned = d0 < a.rot, upper = !PAIRS && sub >= hs;
  const int other = lane + (upper ? -hs : hs);    // lane that holds the other member of the pairs
  float c[8], s[8];
  if (turned) {
    const int i0 = PAIRS ? d0 >> 1 : (upper ? d0 - half : d0);
#pragma unroll
    for (int j = 0; j < (PAIRS ? 4 : 8); ++j) {
      c[j] = cs[wave][0][i0 + j];
      s[j] = cs[wave][1][i0 + j];
      if (upper) s[j] = -s[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) { c[j] = 1.0f; s[j] = 0.0f; }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    wq[j] = NORM && a.wq ? a.wq[d0 + j] : 1.0f;
    wk[j] = NORM && a.wk ? a.wk[d0 + j] : 1.0f;
  }
  // two groups of heads in flight
  const int heads = a.n_heads + a.n_kv_heads;
  const int step = (int)gridDim.y * wpt * HPW;
  auto in_of = [&](int h) {
    const bool key = h >= a.n_heads;
    const int hc = h < heads ? (key ? h - a.n_heads : h) : 0;      // (past the last head: the first query's, never stored)
    return (key && h < heads ? (const uint16_t*)a.K + t * a.ldk : (const uint16_t*)a.Q + t * a.ldq) + (int64_t)hc * DH + d0;
  };
  auto one = [&](int h, uint4 raw) {
    const bool key = h >= a.n_heads;
    u16x8 v = __builtin_bit_cast(u16x8, raw);
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = T::to_float(v[j]);
    if constexpr (NORM) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(u[j], u[j], ss);
#pragma unroll
      for (int off = LPH / 2; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
      const float inv = 1.0f / sqrtf(ss * (1.0f / DH) + a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = u[j] * inv * (key ? wk[j] : wq[j]);
    }
    float o[8];
    if constexpr (PAIRS) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[2 * j] = u[2 * j] * c[j] - u[2 * j + 1] * s[j];
        o[2 * j + 1] = u[2 * j + 1] * c[j] + u[2 * j] * s[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = u[j] * c[j] - __shfl(u[j], other & 63, 64) * s[j];
    }
    if (h >= heads) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = T::from_float(turned ? o[j] : u[j]);
    uint16_t* out = key ? (uint16_t*)a.Ko + t * a.ldko + (int64_t)(h - a.n_heads) * DH : (uint16_t*)a.Qo + t * a.ldqo + (int64_t)h * DH;
    store16(out + d0, __builtin_bit_cast(uint4, v), nts);
  };
  int h0 = ((int)blockIdx.y * wpt + wave % wpt) * HPW + lane / LPH;
  for (; h0 - lane / LPH + step < heads; h0 += 2 * step) {
    const uint4 x = load16<NT>(in_of(h0)), y = load16<NT>(in_of(h0 + step));
    one(h0, x);
    one(h0 + step, y);
  }
  if (h0 - lane / LPH < heads) one(h0, load16<NT>(in_of(h0)));
#endif
}

hipError_t launch_qk_norm_rope(const QkRopeArgs& a, hipStream_t stream) {
  const int heads = a.n_heads + a.n_kv_heads;
  ProfScope ps("qk_norm_rope", stream, 4.0 * (double)a.n_tok * heads * a.head_dim);
  const int groups = (int)ceil_div((int64_t)heads * a.head_dim, 512);
  // a wave takes all heads of a token where the tokens alone fill the chip, otherwise a share of them
  const int wpt = a.n_tok >= 8192 ? 1 : 4;
  unsigned gy = 1;
  if (wpt == 4) {
    const int64_t most = ceil_div(groups, 4), want = ceil_div(2048, a.n_tok);
    gy = (unsigned)(want < most ? want : most);
  }
  const dim3 grid((unsigned)ceil_div(a.n_tok, 4 / wpt), gy);
  const double bytes = 2.0 * (double)a.n_tok * heads * a.head_dim;
  const bool nt = streams_past(2.0 * bytes), nts = nt && outgrows_cache(bytes);
  auto go = [&](auto kern) { kern<<<grid, 256, 0, stream>>>(a, wpt, nts); };
  auto form = [&](auto t, auto dh) {
    using T = decltype(t);
    constexpr int DH = decltype(dh)::value;
    auto norm = [&](auto past) {
      constexpr bool NT = decltype(past)::value;
      if (a.interleaved) a.norm ? go(qk_norm_rope_kernel<T, DH, true, true, NT>) : go(qk_norm_rope_kernel<T, DH, true, false, NT>);
      else a.norm ? go(qk_norm_rope_kernel<T, DH, false, true, NT>) : go(qk_norm_rope_kernel<T, DH, false, false, NT>);
    };
    if (nt) norm(std::true_type{});
    else norm(std::false_type{});
  };
  auto width = [&](auto t) {
    if (a.head_dim == 64) form(t, std::integral_constant<int, 64>{});
    else if (a.head_dim == 128) form(t, std::integral_constant<int, 128>{});
    else form(t, std::integral_constant<int, 256>{});
  };
  a.bf16 ? width(BF16{}) : width(F16{});
  return hipGetLastError();
}

}  // namespace tlq
