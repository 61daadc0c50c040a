// Queries and keys of a decoder block: normalised for each head and rotated by their position, in one pass.
#include <type_traits>

#include "common.h"

namespace tlq {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

#if defined(__HIP_DEVICE_COMPILE__)
template <int CTRL, int BANKS = 0xf>
__device__ __forceinline__ float dpp(float old, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, 0xf, BANKS, true));
}
// v and lane ^ 16's, as {of the even row of 16, of the odd one} (in assembly because the builtin's two results come out as one;
// the wait states are what the swap needs behind the write of its operands)
__device__ __forceinline__ void both_rows(float v, float& even, float& odd) {
  even = odd = v;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(even), "+v"(odd));
}
// sum over the N lanes of a head, in all of them
template <int N>
__device__ __forceinline__ float head_sum(float v) {
  v += dpp<0xB1>(0.0f, v);          // lane ^ 1
  v += dpp<0x4E>(0.0f, v);          // lane ^ 2
  v += dpp<0x141>(0.0f, v);         // the other four of eight
  if constexpr (N >= 16) v += dpp<0x140>(0.0f, v);      // the other eight of sixteen
  if constexpr (N >= 32) {
    float a, b;
    both_rows(v, a, b);
    v = a + b;
  }
  return v;
}
// the value of the lane half a head (N / 2 lanes) away
template <int N>
__device__ __forceinline__ float half_head(float v, bool upper) {
  if constexpr (N == 8) return dpp<0x114, 0xa>(dpp<0x104, 0x5>(0.0f, v), v);      // four up for the lower, four down for the upper
  else if constexpr (N == 16) return dpp<0x128>(0.0f, v);
  else {
    float a, b;
    both_rows(v, a, b);
    return upper ? a : b;
  }
}
#endif

// u = x / sqrt(mean x^2 + eps) * w over the head_dim channels of a head, then the pair (u_a, u_b) turned by
// pos * inv_freq[i].  DH / 8 lanes hold a head, eight channels each, so a wave has 512 / DH heads of one token at a time, two
// groups of them in flight.  The angles belong to the token: a wave computes each cosine and sine once (a lane one or two
// of them, through LDS) and uses them for all heads it takes.  Angles are reduced to a fraction of a turn in double: at
// position 2^31 a float product would be off by whole turns.
// FORM: pairs half a head apart (their lanes trade by lane permutations), half of fewer rotated channels (by LDS), neighbours.
// Bound by the bytes of Q and K, read and written once: 40,800 tokens x 80 heads of 128 332 - 335 us one launch after the other, 337
// - 351 under the profiler, 4.8 - 5.0 TB/s where a copy of as many bytes reaches 3.9 - 5.1; by latency for few tokens: 16 x 40
// heads 5.0 us.
enum { kHalfHead, kHalfRot, kNeighbours };
// AXES: a token has up to four positions and a frequency turns by that of its axis.  The positions are one load more before the
// angles, beside which the frequencies' axes come: 16 x 40 heads 5.4 us, with one axis 5.1; 40,800 x 80 heads 343 and 345.
template <typename T, int DH, int FORM, bool AXES>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkRopeArgs a, int wpt, bool nts) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPH = DH / 8, HPW = 64 / LPH;
  constexpr bool PAIRS = FORM == kNeighbours;
  __shared__ __attribute__((aligned(16))) float cs[4][2][DH / 2];
  const int lane = threadIdx.x & 63, sub = lane & (LPH - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = (int64_t)blockIdx.x * (4 / wpt) + wave / wpt;
  if (t >= a.n_tok) return;                       // (no barrier below)
  const int half = a.rot >> 1;
  {
    double p = 0.0;
    int at[4];
    if constexpr (!AXES) p = (double)a.pos[t];
    else {
#pragma unroll
      for (int x = 0; x < 4; ++x) at[x] = a.pos[(x < a.n_axes ? x : 0) * a.ld_pos + t];
    }
    for (int i = lane; i < half; i += 64) {
      if constexpr (AXES) {
        const int x = a.axis[i];
        p = (double)(x <= 0 ? at[0] : x == 1 || a.n_axes == 2 ? at[1] : x == 2 || a.n_axes == 3 ? at[2] : at[3]);
      }
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
  const int other = (lane + (upper ? -hs : hs)) & 63;      // lane that holds the other member of the pairs
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
    wq[j] = a.wq ? a.wq[d0 + j] : 1.0f;
    wk[j] = a.wk ? a.wk[d0 + j] : 1.0f;
  }
  const int heads = a.n_heads + a.n_kv_heads;
  const int step = (int)gridDim.y * wpt * HPW;
  auto fetch = [&](int h) {
    const bool key = h >= a.n_heads;
    const int hc = h < heads ? (key ? h - a.n_heads : h) : 0;      // (past the last head: the first query's, never stored)
    const uint16_t* p = (key && h < heads ? (const uint16_t*)a.K + t * a.ldk : (const uint16_t*)a.Q + t * a.ldq) + (int64_t)hc * DH + d0;
    return *reinterpret_cast<const uint4*>(p);
  };
  auto one = [&](int h, uint4 raw) {
    const bool key = h >= a.n_heads;
    u16x8 v = __builtin_bit_cast(u16x8, raw);
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = T::to_float(v[j]);
    if (a.norm) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(u[j], u[j], ss);
      float mean = head_sum<LPH>(ss) * (1.0f / DH) + a.eps;
      // (bf16 heads whose squares are no floats, beside ordinary ones of the wave: taken times a power of two; what is not
      // finite stays so)
      const bool fits = mean >= 1e-30f && mean <= 1e37f;
      if (__builtin_expect(__any(!fits), 0)) {
        const float times = fits ? 1.0f : mean < 1e-30f ? 0x1p100f : 0x1p-80f;
        ss = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          u[j] *= times;
          ss = __builtin_fmaf(u[j], u[j], ss);
        }
        mean = head_sum<LPH>(ss) * (1.0f / DH) + a.eps * times * times;
      }
      const float inv = __builtin_amdgcn_rsqf(mean);
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
      for (int j = 0; j < 8; ++j) {
        const float w = FORM == kHalfHead ? half_head<LPH>(u[j], upper) : __shfl(u[j], other, 64);
        o[j] = u[j] * c[j] - w * s[j];
      }
    }
    if (h >= heads) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = T::from_float(FORM == kHalfHead || turned ? o[j] : u[j]);
    uint16_t* out = key ? (uint16_t*)a.Ko + t * a.ldko + (int64_t)(h - a.n_heads) * DH : (uint16_t*)a.Qo + t * a.ldqo + (int64_t)h * DH;
    store16(out + d0, __builtin_bit_cast(uint4, v), nts);
  };
  int h0 = ((int)blockIdx.y * wpt + wave % wpt) * HPW + lane / LPH;
  for (; h0 - lane / LPH + step < heads; h0 += 2 * step) {
    const uint4 x = fetch(h0), y = fetch(h0 + step);
    one(h0, x);
    one(h0 + step, y);
  }
  if (h0 - lane / LPH < heads) one(h0, fetch(h0));
#endif
}

hipError_t launch_qk_norm_rope(const QkRopeArgs& a, hipStream_t stream) {
  const int heads = a.n_heads + a.n_kv_heads;
  ProfScope ps("qk_norm_rope", stream, 4.0 * (double)a.n_tok * heads * a.head_dim);
  const int groups = (int)ceil_div((int64_t)heads * a.head_dim, 512);
  // a wave takes all heads of a token where the tokens alone fill the chip, otherwise a share of them (80 heads of 128, us a
  // wave and four a token: 40,800 tokens 355 454, 10,000 91 110)
  const int wpt = a.n_tok >= 4096 ? 1 : 4;
  unsigned gy = 1;
  if (wpt == 4) {
    const int64_t most = ceil_div(groups, 4), want = ceil_div(2048, a.n_tok);
    gy = (unsigned)(want < most ? want : most);
  }
  const dim3 grid((unsigned)ceil_div(a.n_tok, 4 / wpt), gy);
  const double bytes = 2.0 * (double)a.n_tok * heads * a.head_dim;
  const bool nts = streams_past(2.0 * bytes) && outgrows_cache(bytes);      // (loads past the caches: the same time)
  auto go = [&](auto kern) { kern<<<grid, 256, 0, stream>>>(a, wpt, nts); };
  auto form = [&](auto t, auto dh) {
    using T = decltype(t);
    constexpr int DH = decltype(dh)::value;
    auto axes = [&](auto many) {
      constexpr bool AXES = decltype(many)::value;
      if (a.interleaved) go(qk_norm_rope_kernel<T, DH, kNeighbours, AXES>);
      else if (a.rot == DH) go(qk_norm_rope_kernel<T, DH, kHalfHead, AXES>);
      else go(qk_norm_rope_kernel<T, DH, kHalfRot, AXES>);
    };
    a.axis && a.n_axes > 1 ? axes(std::true_type{}) : axes(std::false_type{});
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
