// New keys and values into the pages of a 4-bit cache, and what a cache holds as 16-bit rows.
#include <type_traits>
#include <utility>

#include "kv4.h"

namespace tlq {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct Kv4CacheDev {
  const uint16_t *K, *V; uint16_t *Ko, *Vo; int64_t ldk, ldv, n_tok;      // rows in, or rows out
  tlq_kv_batch b; tlq_kv_cache c; Kv4Dev d;      // (c: sizes)
};

#if defined(__HIP_DEVICE_COMPILE__)
// A piece of a thread: eight tokens at a multiple of eight, eight channels.  DH / 8 lanes have the channels of a head, four of them
// a group that shares steps.
struct Kv4Piece {
  KvSeq q; int h, d8;          // head, channels 8 d8 and on
  int64_t p0, row0;            // position of the piece's first token (negative before the sequence), its row (may lie outside the rows)
  int lo, hi;                  // of its eight tokens those that are rows of the call
  int id;                      // their page, or -1
  int in_page;                 // of token 0
};
template <int DH>
__device__ __forceinline__ bool kv4_piece(const Kv4CacheDev& a, Kv4Piece& p) {
  constexpr int LPH = DH / 8, EIGHTS = 64 / LPH;
  const int lane = threadIdx.x & 63, wave = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), s = blockIdx.y;
  p.d8 = lane % LPH;
  p.h = wave % a.c.n_kv_heads;
  p.q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  p.p0 = ((int64_t)(p.q.first >> 3) + wave / a.c.n_kv_heads * EIGHTS + lane / LPH) * 8;
  p.row0 = p.q.row0 + p.p0 - p.q.first;
  p.lo = p.q.first > p.p0 ? (int)(p.q.first - p.p0) : 0;
  const int64_t left = (int64_t)p.q.first + p.q.n_new - p.p0;
  p.hi = left < 8 ? (int)left : 8;
  if (p.lo >= p.hi) return false;
  p.in_page = (int)p.p0 & (a.c.page - 1);
  p.id = p.p0 >= 0 && p.p0 < p.q.len ? kv_page(a.b, a.c, s, (int)p.p0 / a.c.page) : -1;
  return true;
}
template <typename Fn, int... E>
__device__ __forceinline__ void static_for8(Fn&& f, std::integer_sequence<int, E...>) { (f(std::integral_constant<int, E>{}), ...); }
template <typename Fn>
__device__ __forceinline__ void static_for8(Fn&& f) { static_for8(f, std::make_integer_sequence<int, 8>{}); }
template <int CTRL>
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {      // with a lane of the same four
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
  return o > v ? o : v;
}
template <typename T> struct Kv4Odd;      // magnitudes (their bits) from which on a group has a number that is not finite, or more than
template <> struct Kv4Odd<F16> { static constexpr uint32_t bits = 0x7c00; };        // seven of the largest steps
template <> struct Kv4Odd<BF16> { static constexpr uint32_t bits = 0x4780; };
// The four bits of a code.  x / step is k + 1/2 exactly or at least 2^-13 away from it: both have few bits (x at least 2^-6 steps: 11
// and 8).  So the product with the reciprocal, off by 1.5 ulp, is brought to a multiple of 2^-16 beside 192, which restores the
// ties and crosses none, and rounded half to even beside 1.5 * 2^23, where the low bits are the code's + 8.
constexpr float kBeside = 192.0f, kCodeAt = 12582920.0f - 192.0f;
constexpr uint32_t kCodeBits = 0x4b400000u;      // what stands in front of them
__device__ __forceinline__ uint32_t kv4_code(float x, float rd) {
  return __builtin_bit_cast(uint32_t, __builtin_fmaf(x, rd, kBeside) + kCodeAt);
}
__device__ __forceinline__ uint32_t kv4_code_any(float x, float rd) {      // also beyond the steps and of NaN
  const float t = __builtin_amdgcn_fmed3f(__builtin_fmaf(x, rd, kBeside), kBeside - kKv4Top, kBeside + kKv4Top);
  return __builtin_bit_cast(uint32_t, (x != x ? kBeside : t) + kCodeAt);
}
// what the fronts of eight codes come to when each is shifted to its place and all are added
constexpr uint32_t kv4_fronts() {
  uint32_t f = 0;
  for (int e = 0; e < 8; ++e) f += kCodeBits << kv4_shift(e);
  return f;
}
#endif

// A token's step for 32 channels is that of its largest value; nothing else has a part in it, so pieces need no meeting but
// that of four lanes.  V's words hold eight tokens of a channel: a piece has all of them, and takes those that are not new from
// memory.  A block's waves have neighbouring heads, whose rows lie side by side.  Bound by bytes: 16 x 613 tokens x 32 heads of 128 in
// pages of 32 48 us, 4.3 TB/s of rows in and codes out (a copy reaches 4.8); by latency for single tokens, 64 x 8 heads 4.6 us.  K and V
// as kernels' bodies of their own, whose registers have constant numbers, and row loads that do not wait for the table: 65 -> 48;
// two instructions a code in place of eight: 75 -> 69 before that.
template <typename T, int DH, bool VAL>
__device__ __forceinline__ void kv4_append_piece(const Kv4CacheDev& a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NG = DH / kKv4Group;
  Kv4Piece p;
  if (!kv4_piece<DH>(a, p)) return;
  const int64_t ld = VAL ? a.ldv : a.ldk;
  const uint16_t* x = (VAL ? a.V : a.K) + p.row0 * ld + p.h * DH + p.d8 * 8;
  // (rows of the call, whether they have a page or not: their loads do not wait for the table)
  uint4 raw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e >= p.lo && e < p.hi) raw[e] = *reinterpret_cast<const uint4*>(x + e * ld);
  if (p.id < 0) return;
  if (p.q.len - p.p0 < p.hi) p.hi = (int)(p.q.len - p.p0);      // (tokens beyond the bounds)
  if (p.lo >= p.hi) return;
  const int64_t slot = (int64_t)p.id * a.c.n_kv_heads + p.h;
  const bool whole = p.lo == 0 && p.hi == 8, first = (p.d8 & 3) == 0;
  const uint32_t words = (uint32_t)a.c.page / 8;
  uint32_t* to = VAL ? a.d.v + (slot * DH + p.d8 * 8) * words + p.in_page / 8 : a.d.k + (slot * a.c.page + p.in_page) * (DH / 8) + p.d8;
  uint16_t* at = VAL ? a.d.v_step + (slot * NG + p.d8 / 4) * a.c.page + p.in_page : a.d.k_step + (slot * a.c.page + p.in_page) * NG + p.d8 / 4;
  uint32_t old[8];
  if (VAL && !whole) {
#pragma unroll
    for (int j = 0; j < 8; ++j) old[j] = to[j * words];
  }
  uint32_t word[8];      // of K: a token's eight channels, of V: a channel's eight tokens
  uint16_t step[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) word[j] = 0;
  auto row = [&](auto ec, auto all) __attribute__((always_inline)) {      // all: numbers of every kind
    constexpr int e = decltype(ec)::value;
    constexpr bool ALL = decltype(all)::value;
    const uint32_t w[4] = {raw[e].x, raw[e].y, raw[e].z, raw[e].w};
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = T::to_float((uint16_t)(w[j >> 1] >> ((j & 1) * 16)));
    uint32_t m = 0;
    if constexpr (ALL) {      // the largest finite one
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = (w[j >> 1] >> ((j & 1) * 16)) & 0x7fffu;
        m = __builtin_isfinite(f[j]) && b > m ? b : m;
      }
    } else {
      u16x2 m2 = {0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, w[j] & 0x7fff7fffu));
      m = m2[0] > m2[1] ? m2[0] : m2[1];
    }
    m = quad_max<0x4E>(quad_max<0xB1>(m));
    // a seventh: one correction step on the product with the reciprocal is the quotient (as in the weights' quantiser)
    const float most = fmaxf(T::to_float((uint16_t)m), kRangeFloor), seventh = 1.0f / kKv4Top, q0 = most * seventh;
    const float wide = BF16::to_float(BF16::from_float(__builtin_fmaf(__builtin_fmaf(-q0, kKv4Top, most), seventh, q0)));
    step[e] = F16::from_float(fminf(wide, kKv4Most));
    const float rd = __builtin_amdgcn_rcpf(F16::to_float(step[e]));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t n = ALL ? kv4_code_any(f[j], rd) : kv4_code(f[j], rd);
      if constexpr (VAL) word[j] += n << kv4_shift(e);
      else word[e] += n << kv4_shift(j);
    }
  };
  // whether a row has a number that is not finite, or that the steps do not reach
  uint32_t fronts = 0, mask = 0;
  static_for8([&](auto ec) __attribute__((always_inline)) {
    constexpr int e = decltype(ec)::value;
    if (e < p.lo || e >= p.hi) return;
    u16x2 m2 = __builtin_elementwise_max(__builtin_bit_cast(u16x2, raw[e].x & 0x7fff7fffu), __builtin_bit_cast(u16x2, raw[e].y & 0x7fff7fffu));
    m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, raw[e].z & 0x7fff7fffu));
    m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, raw[e].w & 0x7fff7fffu));
    if (__builtin_expect(__any(m2[0] >= Kv4Odd<T>::bits || m2[1] >= Kv4Odd<T>::bits), 0)) row(ec, std::true_type{});
    else row(ec, std::false_type{});
    if constexpr (VAL) {
      mask |= 15u << kv4_shift(e);
      fronts += kCodeBits << kv4_shift(e);
    }
  });
  if constexpr (VAL) {
    if (whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j * words] = word[j] - kv4_fronts();
      if (first)
        *reinterpret_cast<uint4*>(at) = make_uint4(step[0] | (uint32_t)step[1] << 16, step[2] | (uint32_t)step[3] << 16,
                                                   step[4] | (uint32_t)step[5] << 16, step[6] | (uint32_t)step[7] << 16);
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j * words] = (old[j] & ~mask) | (word[j] - fronts);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (first && e >= p.lo && e < p.hi) at[e] = step[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= p.lo && e < p.hi) to[e * (DH / 8)] = word[e] - kv4_fronts();
    // the four lanes of a group write steps of two tokens each
    const int j = p.d8 & 3;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const uint16_t mine = j < 2 ? (j == 0 ? step[e] : step[e + 1]) : (j == 2 ? step[e + 2] : step[e + 3]);
      if (e + j >= p.lo && e + j < p.hi) at[(e + j) * NG] = mine;
    }
  }
#endif
}
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4CacheDev a) {
  if (blockIdx.z) kv4_append_piece<T, DH, true>(a);
  else kv4_append_piece<T, DH, false>(a);
}

// The other way: halves as the attention makes them, V's turned back by permutations.  16 x 613 tokens x 32 heads of 128 48 us behind
// other work, 33 right behind their append, whose codes the caches still hold.
template <typename T, int DH, bool VAL>
__device__ __forceinline__ void kv4_read_piece(const Kv4CacheDev& a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NG = DH / kKv4Group;
  Kv4Piece p;
  if (!kv4_piece<DH>(a, p)) return;
  const int64_t ld = VAL ? a.ldv : a.ldk;
  uint16_t* x = (VAL ? a.Vo : a.Ko) + p.row0 * ld + p.h * DH + p.d8 * 8;
  const int64_t slot = (int64_t)(p.id < 0 ? 0 : p.id) * a.c.n_kv_heads + p.h;
  const int there = p.id < 0 ? 0 : p.q.len - p.p0 < 8 ? (int)(p.q.len - p.p0) : 8;      // tokens of the eight that there are
  const Kv4Bits bits = kv4_bits();
  uint4 half[8];      // of K: a token's eight channels, of V: a channel's eight tokens
  if constexpr (!VAL) {
    const int64_t token = slot * a.c.page + p.in_page;
    uint32_t word[8], step[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= p.lo && e < p.hi) {
        word[e] = a.d.k[(token + e) * (DH / 8) + p.d8];
        step[e] = a.d.k_step[(token + e) * NG + p.d8 / 4];
      }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= p.lo && e < p.hi) {
        const uint32_t s = step[e] | step[e] << 16;
        half[e] = kv4_values(word[e], bits, s, s, s, s);
      }
  } else {
    const uint32_t* from = a.d.v + ((slot * DH + p.d8 * 8) * a.c.page + p.in_page) / 8;
    const uint4 s = *reinterpret_cast<const uint4*>(a.d.v_step + (slot * NG + p.d8 / 4) * a.c.page + p.in_page);
    uint32_t word[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) word[j] = from[(int64_t)j * (a.c.page / 8)];
#pragma unroll
    for (int j = 0; j < 8; ++j) half[j] = kv4_values(word[j], bits, s.x, s.y, s.z, s.w);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e < p.lo || e >= p.hi) continue;
    uint32_t o[4];
    if constexpr (!VAL) {
      o[0] = half[e].x; o[1] = half[e].y; o[2] = half[e].z; o[3] = half[e].w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 &u = half[2 * j], &v = half[2 * j + 1];
        const uint32_t c = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w, d = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        o[j] = __builtin_amdgcn_perm(d, c, e & 1 ? 0x07060302u : 0x05040100u);
      }
    }
    if constexpr (std::is_same<T, BF16>::value) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        o[j] = (uint32_t)BF16::from_float(F16::to_float((uint16_t)o[j])) | (uint32_t)BF16::from_float(F16::to_float((uint16_t)(o[j] >> 16))) << 16;
    }
    if (e >= there) o[0] = o[1] = o[2] = o[3] = 0;
    *reinterpret_cast<uint4*>(x + e * ld) = make_uint4(o[0], o[1], o[2], o[3]);
  }
#endif
}
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4CacheDev a) {
  if (blockIdx.z || !a.Ko) kv4_read_piece<T, DH, true>(a);
  else kv4_read_piece<T, DH, false>(a);
}

// eights of tokens that a sequence's new ones can lie in, wherever they begin; a wave has 512 / head_dim of them for a head
int64_t kv4_cache_blocks(int64_t n_tok, const tlq_kv_batch& b, const tlq_kv4_cache& c) {
  const int64_t eights = ((b.max_new < n_tok ? b.max_new : n_tok) + 14) / 8;
  return ceil_div(c.n_kv_heads * ceil_div(eights, 512 / c.head_dim), 4);
}

hipError_t launch_kv4_append(const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch& b,
                             const tlq_kv4_cache& c, bool bf16, hipStream_t stream) {
  ProfScope ps("kv4_append", stream, 5.125 * (double)n_tok * c.n_kv_heads * c.head_dim);
  Kv4CacheDev a{};
  a.K = (const uint16_t*)K; a.V = (const uint16_t*)V; a.ldk = ldk; a.ldv = ldv; a.n_tok = n_tok;
  a.b = b; a.c = kv4_sizes(c); a.d = {c.k, c.k_step, c.v, c.v_step};
  const dim3 grid((unsigned)kv4_cache_blocks(n_tok, b, c), (unsigned)b.n_seq, 2);
  auto pick = [&](auto t) {
    using T = decltype(t);
    if (c.head_dim == 128) kv4_append_kernel<T, 128><<<grid, 256, 0, stream>>>(a);
    else kv4_append_kernel<T, 64><<<grid, 256, 0, stream>>>(a);
  };
  bf16 ? pick(BF16{}) : pick(F16{});
  return hipGetLastError();
}

hipError_t launch_kv4_read(void* K, int64_t ldk, void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch& b, const tlq_kv4_cache& c,
                           bool bf16, hipStream_t stream) {
  ProfScope ps("kv4_read", stream, (K && V ? 5.125 : 2.5625) * (double)n_tok * c.n_kv_heads * c.head_dim);
  Kv4CacheDev a{};
  a.Ko = (uint16_t*)K; a.Vo = (uint16_t*)V; a.ldk = ldk; a.ldv = ldv; a.n_tok = n_tok;
  a.b = b; a.c = kv4_sizes(c); a.d = {c.k, c.k_step, c.v, c.v_step};
  const dim3 grid((unsigned)kv4_cache_blocks(n_tok, b, c), (unsigned)b.n_seq, K && V ? 2 : 1);
  auto pick = [&](auto t) {
    using T = decltype(t);
    if (c.head_dim == 128) kv4_read_kernel<T, 128><<<grid, 256, 0, stream>>>(a);
    else kv4_read_kernel<T, 64><<<grid, 256, 0, stream>>>(a);
  };
  bf16 ? pick(BF16{}) : pick(F16{});
  return hipGetLastError();
}

}  // namespace tlq
