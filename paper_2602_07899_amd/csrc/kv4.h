// What the kernels of the 4-bit cache share: words of eight codes, element e in the four bits from 4 (e / 2) + 16 (e % 2) up.
#pragma once
#include "kv.h"

namespace tlq {

constexpr int kKv4Group = 32;            // channels that share a token's step
constexpr float kKv4Top = 7.0f, kKv4Most = 9344.0f;

// the codes and sizes of a cache for the kernels
struct Kv4Dev { uint32_t* k; uint16_t* k_step; uint32_t* v; uint16_t* v_step; };

// A cache's sizes for what both caches share (the pointers stay null)
inline tlq_kv_cache kv4_sizes(const tlq_kv4_cache& c) {
  tlq_kv_cache s{};
  s.struct_size = sizeof(tlq_kv_cache);
  s.n_kv_heads = c.n_kv_heads; s.head_dim = c.head_dim; s.page = c.page; s.n_pages = c.n_pages;
  return s;
}

__host__ __device__ constexpr int kv4_shift(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

#if defined(__HIP_DEVICE_COMPILE__)
typedef _Float16 kv4_f16x2 __attribute__((ext_vector_type(2)));
// The bits of a pair of codes and what stands in front of them: four bits behind the exponent of 1024 are 1024 + n, four bits higher
// up behind that of 64 are 64 + n.  In registers (as constants of an instruction each would need two of them).
struct Kv4Bits { uint32_t low, high, k1024, k64; };
__device__ __forceinline__ Kv4Bits kv4_bits() {
  Kv4Bits b{0x000f000fu, 0x00f000f0u, 0x64006400u, 0x54005400u};
  asm("" : "+s"(b.low), "+s"(b.high));
  asm("" : "+v"(b.k1024), "+v"(b.k64));
  return b;
}
// pair p (elements 2 p, 2 p + 1) of a word, less eight, as halves
template <int P>
__device__ __forceinline__ kv4_f16x2 kv4_pair(uint32_t w, const Kv4Bits& b) {
  const uint32_t x = P >= 2 ? w >> 8 : w;
  constexpr bool UP = P & 1;
  const uint32_t h = (x & (UP ? b.high : b.low)) | (UP ? b.k64 : b.k1024);
  const kv4_f16x2 off = {(_Float16)(UP ? 72.0f : 1032.0f), (_Float16)(UP ? 72.0f : 1032.0f)};
  return __builtin_bit_cast(kv4_f16x2, h) - off;
}
// eight codes times their steps (pairs, as halves): exact, a step has eight significant bits
__device__ __forceinline__ uint4 kv4_values(uint32_t w, const Kv4Bits& b, uint32_t s0, uint32_t s1, uint32_t s2, uint32_t s3) {
  auto h = [](uint32_t s) { return __builtin_bit_cast(kv4_f16x2, s); };
  return make_uint4(__builtin_bit_cast(uint32_t, kv4_pair<0>(w, b) * h(s0)), __builtin_bit_cast(uint32_t, kv4_pair<1>(w, b) * h(s1)),
                    __builtin_bit_cast(uint32_t, kv4_pair<2>(w, b) * h(s2)), __builtin_bit_cast(uint32_t, kv4_pair<3>(w, b) * h(s3)));
}
#endif

}  // namespace tlq
