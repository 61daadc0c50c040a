// What attention over the 8-bit and over the 4-bit cache share: a launch's plan, queries, the softmax's sums, the joining of splits.
#pragma once
#include <type_traits>

#include "kv.h"

namespace tlq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// r / d for 0 <= r < 2^31, 1 <= d < 2^31, as a product (Granlund and Montgomery, 1994): m = ceil(2^(31+s) / d), s = ceil(log2 d)
struct KvDiv {
  uint32_t m, s, d;
  __device__ __forceinline__ uint32_t of(uint32_t r) const { return __umulhi(r << 1, m) >> s; }
};
inline KvDiv kv_div(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s, d};
}

struct KvAttnDev {
  const uint16_t* Q; int64_t ldq, n_tok; int n_heads, group; KvDiv by_group; float scale2;    // scale * log2(e)
  tlq_kv_batch b; tlq_kv_cache c; int page_bits;
  uint16_t* Out; int64_t ldo;
  int n_splits, chunk;          // keys of a split
  // kv_prompt_kernel: row tiles; pairs of sequence and key head, blocks of a pair, and of the pairs that an XCD has to itself
  int tiles; uint32_t n_pairs, own_blocks, together_bits; KvDiv by_heads, by_work;
  float2* ml; float* acc;       // per (row, head, split): reference and sum; [head_dim] sums of codes
};

// How a call is launched: prompts' tiles of 128 rows or few tiles of 16, splits of the keys, room in the workspace
struct KvPlan { bool prompt; int rows, tiles, n_splits, chunk; size_t acc_at, bytes; };
KvPlan kv_plan(int64_t n_tok, int n_heads, const tlq_kv_batch& b, const tlq_kv_cache& c, bool bits4);      // (sizes are read, no pointer)
KvAttnDev kv_attn_dev(const KvPlan& p, const void* Q, int64_t ldq, int64_t n_tok, int n_heads, float scale, const tlq_kv_batch& b,
                      const tlq_kv_cache& c, void* Out, int64_t ldo, void* workspace, dim3* grid);
hipError_t launch_kv_join(const KvPlan& p, const KvAttnDev& a, bool from_last, bool bf16, hipStream_t stream);

template <int I, int N, typename Fn>
__device__ __forceinline__ void static_for(Fn&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

#if defined(__HIP_DEVICE_COMPILE__)
constexpr float kTop = 7.0f, kRaise = 15.0f;      // exponents of the largest weight: when the reference is set, at most
// sum of eight weights (rounded already) and c
__device__ __forceinline__ float add_weights(f16x8 w, float c) {
  const f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_fdot2(f16x2{w[2 * i], w[2 * i + 1]}, one, c, false);
  return c;
}
// the largest of a value that lane ^ 16 and lane ^ 32 hold (as in block.hip: the builtins' two results come out as one; the wait
// states are what the swaps need behind the write of an operand)
__device__ __forceinline__ float column_max(float v) {
  float a = v, b = v;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  a = b = fmaxf(a, b);
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// A denominator times 2^d, d <= 0.  Steps of values may lie further apart than floats have exponents: where 2^d has none left the
// denominator takes the way in two.  With f = 2^d at hand where a launch is a chain of few of them (1200 keys x 32 9.9 us, the other
// form 10.0), without a branch between the products of prompts (16 of up to 1200 tokens 343 us, the other form 348).
__device__ __forceinline__ float lower_sum(float l, float d, float f) {
  const bool far = l != 0.0f && d < -100.0f;
  float r = l * f;
  if (__builtin_expect(__any(far), 0)) r = far ? l * 0x1p-100f * exp2_fast(d + 100.0f) : r;
  return r;
}
__device__ __forceinline__ float lower_sum(float l, float d) {
  const float c = fmaxf(d, -100.0f);
  return l * exp2_fast(c) * exp2_fast(d - c);      // (the last is one down to there)
}

// A query with an infinity or NaN is not to end as a row without keys (all of its scores -inf, or none above the maximum so far):
// a lane that holds such a number makes a NaN of it, and with it the products with every key.
template <int N>
__device__ __forceinline__ void mark_queries(f16x8 (&qf)[N]) {
  const f16x2 zero = {(_Float16)0.0f, (_Float16)0.0f};
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; e += 2) t = __builtin_amdgcn_fdot2(f16x2{qf[i][e], qf[i][e + 1]}, zero, t, false);
  qf[0][0] = t == t ? qf[0][0] : (_Float16)t;
}
__device__ __forceinline__ uint32_t column_max_bits(uint32_t v) {      // as column_max, of unsigned numbers
  uint32_t a = v, b = v;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  a = b = a > b ? a : b;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return a > b ? a : b;
}
// A lane's channels of its query as halves, eight at a time and STEP apart (negated if asked); the factor that undoes their
// prescale.  Lanes lane ^ 16 and lane ^ 32 hold the other channels of the same query.  bf16 in pairs as they lie takes 250 instructions
// for 32 rows, element by element 600: 1200 keys x 32 9.8 us and 10.2, 16 prompts of 1200 tokens x 40 over a 4-bit cache 356 and 359.
template <typename T, int N, int STEP>
__device__ __forceinline__ float load_queries(const uint16_t* p, f16x8 (&qf)[N], bool negate) {
  uint4 raw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) raw[i] = *reinterpret_cast<const uint4*>(p + STEP * i);
  if constexpr (std::is_same<T, F16>::value) {
    const uint32_t sign = negate ? 0x80008000u : 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      qf[i] = __builtin_bit_cast(f16x8, make_uint4(raw[i].x ^ sign, raw[i].y ^ sign, raw[i].z ^ sign, raw[i].w ^ sign));
    mark_queries(qf);
    return 1.0f;
  }
  u16x2 top2 = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
  }
  const uint32_t top = column_max_bits(top2[0] > top2[1] ? top2[0] : top2[1]);
  // exponent field of the largest -> 127 + 14; rows of zeros and subnormals keep factors that are finite, infinities stay
  int k = 141 - (int)(top >> 7);
  k = k > 126 ? 126 : k;
  const float up = __builtin_bit_cast(float, (uint32_t)(127 + k) << 23 | (negate ? 0x80000000u : 0));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      qf[i][2 * e] = (_Float16)(__builtin_bit_cast(float, w[e] << 16) * up);
      qf[i][2 * e + 1] = (_Float16)(__builtin_bit_cast(float, w[e] & 0xffff0000u) * up);
    }
  }
  if (top >= 0x7f80u) qf[0][0] = (_Float16)__builtin_nanf("");      // (as mark_queries; the row's other lanes may)
  return __builtin_bit_cast(float, (uint32_t)(127 - k) << 23);
}
#endif

}  // namespace tlq
