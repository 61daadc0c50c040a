// Causal attention over an 8-bit cache in pages.
//
// Mathematics.  Key j of a head is kcode_j * ks(j), value j is vcode_j * vs(j), with one step ks, vs for each page and head.
// With z_j = scale * log2(e) * ks(j) * (q . kcode_j) + log2(vs(j)) and any reference m,
//   out = sum_j 2^(z_j - m) vcode_j  /  sum_j 2^(z_j - m) / vs(j):
// the values' step goes into the exponent for nothing, so that the codes enter the second product as they are and the
// weights that are rounded to 16 bits are those of the contributions, not of the probabilities - a page of small values
// (a first token's) cannot push the rest below the smallest half.  m, the row's reference, is 7 below the largest z when it
// is set, and is set again when a z lies 15 above it: weights stay between 2^15 and, as normal halves, 2^-21 of the largest
// at least (with the largest at 1, 2^-14: over 10^5 keys what falls below would show), and sums are rescaled a few times a
// row instead of at every new maximum.  The denominator sums the rounded weights, in 32 bits: where one key has nearly all
// of the weight its rounding cancels.  But a page whose step lies far below the others' has small weights 2^(z - m) whatever
// its probabilities are, and in the denominator they are divided by that step: such halves would be subnormal or zero.  Where a
// lane's page has a step below 2^-3 of those that the reference was set among, and the largest of the lane's 16 weights is
// below 2^-7, it sums sum_j 2^(scale log2(e) ks (q . kcode_j) - m) from unrounded exponentials.  What the denominator can lose
// otherwise, next to the roundings to 2^-12: 15 times 2^-25 beside a weight of 2^-7 at least (2^-14 of itself), and 2^-25 a key
// at 2^3 times the reference's step and weight of 2^7, so 2^-29 a key (2^-12 over 131,072 keys, all of them below the
// halves).  Both products run on fp16 matrix instructions whatever x_dtype is: codes are exact in
// fp16; bf16 queries are multiplied with the power of two that brings the largest of the row to [2^14, 2^15).
// The products are transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane owns one query column and P stays in
// registers; values are stored channel by channel so that V^T's rows are read as they lie.
#include <type_traits>

#include "kv.h"

namespace tlq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

// r / d for 0 <= r < 2^31, 1 <= d < 2^31, as a product (Granlund and Montgomery, 1994): m = ceil(2^(31+s) / d), s = ceil(log2 d)
struct KvDiv {
  uint32_t m, s, d;
  __device__ __forceinline__ uint32_t of(uint32_t r) const { return __umulhi(r << 1, m) >> s; }
};
static KvDiv kv_div(uint32_t d) {
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

template <int I, int N, typename Fn>
__device__ __forceinline__ void static_for(Fn&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

#if defined(__HIP_DEVICE_COMPILE__)
constexpr float kSmallStep = 1e-30f;    // (a step of zero: its page's values count as zeros, its keys in the sum as ever)
constexpr float kTop = 7.0f, kRaise = 15.0f;      // exponents of the largest weight: when the reference is set, at most
constexpr float kNear = 3.0f, kLow = 7.0f;        // binary orders below the reference's step, below a weight of one (see above)
// sum of eight weights (rounded already) and c
__device__ __forceinline__ float add_weights(f16x8 w, float c) {
  const f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_fdot2(f16x2{w[2 * i], w[2 * i + 1]}, one, c, false);
  return c;
}
// four codes -> four halves: byte + 128 behind the exponent of 1024, less 1152
__device__ __forceinline__ void widen_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off);
  hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off);
}
__device__ __forceinline__ f16x8 widen_codes8(uint32_t a, uint32_t b) {
  uint4 v;
  widen_codes(a, v.x, v.y);
  widen_codes(b, v.z, v.w);
  return __builtin_bit_cast(f16x8, v);
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
// A lane's channels of its query as halves, eight at a time and STEP apart (negated if asked); the factor that undoes their
// prescale.  Lanes lane ^ 16 and lane ^ 32 hold the other channels of the same query.
template <typename T, int N, int STEP>
__device__ __forceinline__ float load_queries(const uint16_t* p, f16x8 (&qf)[N], bool negate) {
  u16x8 raw[N];
  const unsigned short sign = negate ? 0x8000 : 0;
#pragma unroll
  for (int i = 0; i < N; ++i) raw[i] = *reinterpret_cast<const u16x8*>(p + STEP * i) ^ sign;
  if constexpr (std::is_same<T, F16>::value) {
#pragma unroll
    for (int i = 0; i < N; ++i) qf[i] = __builtin_bit_cast(f16x8, raw[i]);
    mark_queries(qf);
    return 1.0f;
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = raw[i][e] & 0x7fffu;
      top = a > top ? a : top;
    }
  for (int off = 16; off <= 32; off <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, off, 64);
    top = o > top ? o : top;
  }
  // exponent field of the largest -> 127 + 14; rows of zeros and subnormals keep factors that are finite, infinities stay
  int k = 141 - (int)(top >> 7);
  k = k > 126 ? 126 : k;
  const float up = __builtin_bit_cast(float, (uint32_t)(127 + k) << 23);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) qf[i][e] = (_Float16)(BF16::to_float(raw[i][e]) * up);
  mark_queries(qf);
  return __builtin_bit_cast(float, (uint32_t)(127 - k) << 23);
}
#endif

// The 16 rows of a tile (a query and head each: the heads that share a key head are rows side by side) against one split of
// the keys.  Four waves take 64 keys each in turn and meet in LDS at the end; keys and values go from memory to registers,
// where they are widened: no LDS, no barrier in the loop, the next 64 keys in flight while these are worked on.
// For few rows (see kFewWork), bound by the bytes of the cache: 64 sequences of 4096 - 8192 tokens x 8 key heads of 128, four queries each,
// 158 us, 5.1 TB/s of codes (a large copy reaches 5.06); one of 131,072 x 4 26 us, 5.1 TB/s; one of 1200 x 32 6.9 us, latency.
template <typename T, int DH>
__global__ __launch_bounds__(256, 3) void kv_few_kernel(KvAttnDev a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NS = DH / 32, ND = DH / 16, LW = DH / 64;    // k32 steps of a score, channel tiles, 16-byte pieces of a lane's key
  constexpr int RS = DH + 4;
  __shared__ __attribute__((aligned(16))) float part[4][16][RS];
  __shared__ float2 ml[4][16];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s = blockIdx.z, hk = blockIdx.y;
  const int tile = (int)blockIdx.x / a.n_splits, split = (int)blockIdx.x % a.n_splits;
  const KvSeq q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  const uint32_t rows = (uint32_t)q.n_new * a.group, first_row = (uint32_t)tile * 16;
  if (first_row >= rows) return;
  const uint32_t row = first_row + l16 < rows ? first_row + l16 : rows - 1;
  const int qi = (int)a.by_group.of(row), g = (int)(row - qi * a.group);
  const int pos = q.first + qi;
  const int last = q.first + (int)a.by_group.of(first_row + 15 < rows ? first_row + 15 : rows - 1);      // the tile's latest position
  const int end = last + 1 < q.len ? last + 1 : q.len;
  const int k0 = split * a.chunk;
  if (k0 >= end && a.n_splits > 1) return;
  const int k1 = end - k0 < a.chunk ? end : k0 + a.chunk;

  f16x8 qf[NS];
  const float fac = a.scale2 * load_queries<T, NS, 8>(
      a.Q + (q.row0 + qi) * a.ldq + ((int64_t)hk * a.group + g) * DH + fq * (DH / 4), qf, false);

  f32x4 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref = -INFINITY, l_run = 0.0f;      // the row's reference, this lane's share of its sum
  float quiet = -INFINITY;                  // kNear below the largest step (its logarithm) among the keys that set the reference

  uint4 kr[4][LW], vr[ND];
  float ks = 0.0f, vs = 1.0f;
  bool seen = false;                    // this lane's 16 keys lie in a page that there is
  // The table's entries are fetched a turn before the pages they name (keys behind the last are never seen: any entry will
  // do); an entry outside the pool becomes the first page, in reach and never seen
  const int32_t* row_table = a.b.table + (int64_t)s * a.b.ld_table;
  const int64_t head_bytes = (int64_t)a.c.page * DH;
  const uint32_t page_stride = (uint32_t)a.c.n_kv_heads * a.c.page * DH, n_pages = (uint32_t)a.c.n_pages;
  const int8_t* kp = a.c.k + hk * head_bytes + (l16 & 3) * DH + fq * (DH / 4);
  const int8_t* vp = a.c.v + hk * head_bytes + l16 * a.c.page;
  const int kgroup = (l16 >> 2) * 16, vgroup = fq * 16;
  uint32_t kid = 0, vid = 0;
  auto entry = [&](int key) { return (uint32_t)row_table[(key < k1 ? key : k1 - 1) >> a.page_bits]; };
  auto load_k = [&](int unit) {
    const int8_t* p = kp + (uint64_t)(kid < n_pages ? kid : 0) * page_stride + ((unit + kgroup) & (a.c.page - 1)) * DH;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < LW; ++i) kr[j][i] = *reinterpret_cast<const uint4*>(p + j * 4 * DH + i * 16);
    kid = entry(unit + 256 + kgroup);
  };
  auto load_v = [&](int unit) {
    seen = vid < n_pages;
    const uint32_t id = seen ? vid : 0;
    const int8_t* p = vp + (uint64_t)id * page_stride + ((unit + vgroup) & (a.c.page - 1));
#pragma unroll
    for (int d = 0; d < ND; ++d) vr[d] = *reinterpret_cast<const uint4*>(p + d * 16 * a.c.page);
    const uint64_t slot = (uint64_t)id * a.c.n_kv_heads + hk;
    ks = seen ? a.c.k_step[slot] : 0.0f;
    vs = seen ? fmaxf(a.c.v_step[slot], kSmallStep) : 1.0f;
    vid = entry(unit + 256 + vgroup);
  };

  int unit = k0 + wave * 64;
  if (unit < k1) {
    kid = entry(unit + kgroup);
    vid = entry(unit + vgroup);
    load_k(unit);
    load_v(unit);
  }
  for (; unit < k1; unit += 256) {
    f32x4 sc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const uint4 w = kr[j][i >> 1];
        const f16x8 kf = (i & 1) ? widen_codes8(w.z, w.w) : widen_codes8(w.x, w.y);
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[i], sc[j], 0, 0, 0);
      }
    }
    if (unit + 256 < k1) load_k(unit + 256);
    // lane: keys unit + 16 fq + 4 j + r of its query
    const float f = fac * ks, lg = __builtin_amdgcn_logf(vs), rv = __builtin_amdgcn_rcpf(vs);
    const int limit = seen ? (pos < k1 - 1 ? pos : k1 - 1) - (unit + fq * 16) : -1;    // last visible of the 16
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float z = __builtin_fmaf(sc[j][r], f, lg);
        sc[j][r] = 4 * j + r <= limit ? z : -INFINITY;
        mx = fmaxf(mx, sc[j][r]);
      }
    const float own = mx;
    mx = column_max(mx);
    float per = rv;                       // of the rounded weights' sum, in the denominator
    if (__any(mx > ref + kRaise || lg < quiet)) {
      const float lg_top = column_max(own != -INFINITY ? lg : -INFINITY);
      if (mx > ref + kRaise) {
        const float next = mx - kTop, alpha = exp2_fast(ref - next);       // (0 at the first visible key)
        l_run = lower_sum(l_run, ref - next, alpha);
        ref = next;
        quiet = lg_top - kNear;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] *= alpha;
      }
      if (lg < quiet && own < ref - kLow) {
        const float less = ref + lg;
        per = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) l_run += exp2_fast(sc[e >> 2][e & 3] - less);
      }
    }
    const float from = ref == -INFINITY ? 0.0f : ref;
    f16x8 pf[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = (_Float16)exp2_fast(sc[e >> 2][e & 3] - from);
    l_run = __builtin_fmaf(add_weights(pf[1], add_weights(pf[0], 0.0f)), per, l_run);
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen_codes8(vr[d].x, vr[d].y), pf[0], acc[d], 0, 0, 0);
      acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen_codes8(vr[d].z, vr[d].w), pf[1], acc[d], 0, 0, 0);
    }
    if (unit + 256 < k1) load_v(unit + 256);
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (fq == 0) ml[wave][l16] = make_float2(ref, l_run);
  __syncthreads();
  const float top = fmaxf(fmaxf(ml[0][l16].x, ml[1][l16].x), fmaxf(ml[2][l16].x, ml[3][l16].x));
  const float mine = ref == -INFINITY ? 0.0f : exp2_fast(ref - top);
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<f32x4*>(&part[wave][l16][d * 16 + fq * 4]) = acc[d] * mine;
  __syncthreads();
  // 16 lanes a row, DH / 16 channels each
  constexpr int PER = DH / 16;
  const int r = tid >> 4, d0 = (tid & 15) * PER;
  if (first_row + r >= rows) return;
  float m = -INFINITY, l = 0.0f, o[PER];
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w][r].x);
#pragma unroll
  for (int w = 0; w < 4; ++w)
    l += lower_sum(ml[w][r].y, ml[w][r].x - m, ml[w][r].x == -INFINITY ? 0.0f : exp2_fast(ml[w][r].x - m));      // (NaN stays)
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = (part[0][r][d0 + e] + part[1][r][d0 + e]) + (part[2][r][d0 + e] + part[3][r][d0 + e]);
  const uint32_t oq = a.by_group.of(first_row + r);
  const int64_t token = q.row0 + oq, head = (int64_t)hk * a.group + (first_row + r - oq * a.group);
  if (a.n_splits > 1) {
    const int64_t at = (token * a.n_heads + head) * a.n_splits + split;
    if ((tid & 15) == 0) a.ml[at] = make_float2(m, l);
#pragma unroll
    for (int e = 0; e < PER; e += 4)
      *reinterpret_cast<float4*>(a.acc + at * DH + d0 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
    return;
  }
  const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t w[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) w[e] = T::from_float(o[e] * inv);
  uint16_t* to = a.Out + token * a.ldo + head * DH + d0;
#pragma unroll
  for (int e = 0; e < PER; e += 4)
    *reinterpret_cast<uint2*>(to + e) = make_uint2((uint32_t)w[e] | (uint32_t)w[e + 1] << 16, (uint32_t)w[e + 2] | (uint32_t)w[e + 3] << 16);
#endif
}

// 128 rows of a sequence and key head against one split of the keys, 32 rows a wave, 64 keys a step.  The keys and values of
// a step are widened once for the block on their way into LDS: what comes from memory during one step is written during
// the next into the stage that nobody reads (one barrier a step).  A lane has 16 neighbouring keys of two queries: they lie
// in one page, so its steps are two numbers, and the largest exponent is found on the bare products.
// Bound by the issue of vector instructions (an exponential, a conversion and a fused product for each score, beside them the
// widening) and, where sequences are long, by power: 16 prompts of up to 1200 tokens x 40 heads of 128 343 - 361 us (one launch
// after the other; 380 - 391 under the profiler), 600 - 630 TFLOP/s of what the mask leaves (a quarter more is computed on the
// diagonal's tiles, and a block has only 19 steps at most), 4 of 2400 292 - 303 us, 9600 tokens x 40 heads 1000 - 1033 us, 915 -
// 945 TFLOP/s; a library product of halves reaches 1130.  Sums of unrounded weights in every second page: the first 364 us for
// 343.
// Not kept, us before and with it for the first: 256 rows with eight waves 427 457, staging held in registers by hand no gain;
// P through LDS is not needed, S^T's columns are P^T's.
// All row tiles of a sequence and key head run on one XCD, the longest first, as far as the pairs can be dealt out evenly.
template <typename T, int DH>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void kv_prompt_kernel(KvAttnDev a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NS = DH / 32, ND = DH / 16, CPK = DH / 8;   // k32 steps of a score, channel tiles, 16-byte chunks of a key
  constexpr int KB = DH * 2, VB = 128;                      // bytes of a row of K, of V^T in LDS
  constexpr int STAGE = 64 * KB + DH * VB, LR = DH / 64;    // LR: 16-byte loads of a thread for K, and for V
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // block 8 j + x runs on XCD x.  It has pair x of each eight: 2^together_bits such pairs at a time, then those that are left of
  // them, the longest tiles of all first.  The pairs that are no eight come last, their blocks one XCD after the other.
  const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x, x = block & 7;
  uint32_t j = block >> 3, sh, which;
  if (j < a.own_blocks) {
    const uint32_t own = a.n_pairs >> 3, full = own >> a.together_bits << a.together_bits;
    if (j < full * a.by_work.d) {
      const uint32_t g = a.by_work.of(j >> a.together_bits);
      which = (j >> a.together_bits) - g * a.by_work.d;
      sh = ((g << a.together_bits) + (j & ((1u << a.together_bits) - 1))) * 8 + x;
    } else {
      j -= full * a.by_work.d;
      which = j / (own - full);
      sh = (full + j - which * (own - full)) * 8 + x;
    }
  } else {
    j = (j - a.own_blocks) * 8 + x;
    const uint32_t g = a.by_work.of(j);
    which = j - g * a.by_work.d;
    sh = (a.n_pairs & ~7u) + g;
    if (sh >= a.n_pairs) return;
  }
  const uint32_t turn = a.n_splits == 1 ? which : which / (uint32_t)a.n_splits;
  const int tile = a.tiles - 1 - (int)turn, split = (int)(which - turn * a.n_splits);
  const int s = (int)a.by_heads.of(sh), hk = (int)(sh - s * a.by_heads.d);
  const int k0 = split * a.chunk;
  // Table entries are the same for the whole block (scalar loads, a step before the pages they name are loaded, the first beside the
  // lengths); entries behind the last key are never seen, any will do, and one outside the pool becomes the first page, in
  // reach and never seen.  A step's first key is a multiple of 64, so a page's part of an offset is a scalar.
  const auto row_table = (const __attribute__((address_space(4))) int32_t*)(a.b.table + (int64_t)s * a.b.ld_table);
  uint32_t ids[4];                     // of the next four 16 keys
  auto entries = [&](int unit) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at = (unit + g * 16) >> a.page_bits;
      ids[g] = (uint32_t)row_table[at < a.b.max_pages ? at : a.b.max_pages - 1];
    }
  };
  entries(k0);
  const KvSeq q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  const uint32_t rows = (uint32_t)q.n_new * a.group, first_row = (uint32_t)tile * 128;
  if (first_row >= rows) return;
  auto last_key = [&](uint32_t r) {      // number of keys that rows up to r see
    const int p = q.first + (int)a.by_group.of(r < rows - 1 ? r : rows - 1);
    return p + 1 < q.len ? p + 1 : q.len;
  };
  const int end = last_key(first_row + 127);
  if (k0 >= end && a.n_splits > 1) return;
  const int k1 = end - k0 < a.chunk ? end : k0 + a.chunk;
  const uint32_t wrow = first_row + wave * 32;
  const int wend = wrow < rows ? (last_key(wrow + 31) < k1 ? last_key(wrow + 31) : k1) : 0;    // keys of this wave
  const int wfull = wrow < rows ? last_key(wrow) : 0;                                          // keys that all of its rows see

  f32x4 acc[ND][2];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d][0] = acc[d][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.0f, 0.0f};
  float quiet = -INFINITY;                 // as in kv_few_kernel, the larger of the two columns'

  // what a thread moves: K rows tid / (CPK / 2) and further ones, 16 codes; V channels 16 wave + l16 and 64 further, the 16 keys
  // that it has the scores of.
  const int krow = tid / (CPK / 2), kch = tid % (CPK / 2) * 2, vrow = wave * 16 + l16;
  constexpr int KSTEP = 512 / CPK;                          // rows between a thread's loads of K
  const uint32_t head_bytes = (uint32_t)a.c.page * DH, page_stride = (uint32_t)a.c.n_kv_heads * head_bytes;
  const uint32_t n_pages = (uint32_t)a.c.n_pages, in_page = (uint32_t)a.c.page - 1;
  const int8_t *kp = a.c.k + (uint64_t)hk * head_bytes, *vp = a.c.v + (uint64_t)hk * head_bytes;
  uint32_t koff[LR], voff[LR];
#pragma unroll
  for (int i = 0; i < LR; ++i) {
    koff[i] = ((uint32_t)(krow + i * KSTEP) & in_page) * DH + kch * 8;
    voff[i] = (uint32_t)(vrow + i * 64) * a.c.page + ((uint32_t)(fq * 16) & in_page);
  }
  uint4 kr[LR], vr[LR];
  bool seen = false, seen_next = false;
  float ks = 0.0f, vs = 1.0f, ks_next = 0.0f, vs_next = 1.0f;
  auto load = [&](int unit) {          // (the steps in front: who waits for them waits for what was issued before)
    const uint32_t at = (uint32_t)unit & in_page;
    const uint32_t mine = fq < 2 ? (fq == 0 ? ids[0] : ids[1]) : (fq == 2 ? ids[2] : ids[3]);
    seen_next = mine < n_pages;
    const uint32_t id = seen_next ? mine : 0;
    const uint64_t slot = (uint64_t)id * (uint32_t)a.c.n_kv_heads + (uint32_t)hk;
    ks_next = a.c.k_step[slot];
    vs_next = a.c.v_step[slot];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < LR; ++i) {     // (DH = 128: a wave's rows lie in one group of 16 keys; 64: wave w has group w)
      const int g = DH == 128 ? (wave >> 1) + 2 * i : wave;
      const uint32_t k = g == 0 ? ids[0] : g == 1 ? ids[1] : g == 2 ? ids[2] : ids[3];
      kr[i] = *reinterpret_cast<const uint4*>(kp + ((uint64_t)(k < n_pages ? k : 0) * page_stride + at * DH) + koff[i]);
    }
    const int8_t* p = vp + at + (uint64_t)id * page_stride;
#pragma unroll
    for (int i = 0; i < LR; ++i) vr[i] = *reinterpret_cast<const uint4*>(p + voff[i]);
    entries(unit + 64);
  };
  // Chunk c of a row lies at place(c) ^ key(row), such that neither the eight lanes of a write that are served together (128
  // bytes) nor the sixteen of a read (lanes 0 - 3, 12 - 15, 20 - 27 of 32 and the others, 256 bytes) meet in a bank: sixteen
  // bytes for each row parity and key.  Rows of 256 bytes have the even chunks in front, the others with bits 2 and 3 turned.
  auto kkey = [](int row) { return DH == 128 ? (row >> 4 & 3) * 4 + (row & 3) : (row >> 4 & 1) * 4 + (row & 3); };
  auto kplace = [](int c) { return DH == 128 ? c >> 1 ^ (c & 1) * 12 : c; };
  // one of a thread's 4 LR pieces of the next stage: eight codes, widened
  auto stage = [&](unsigned char* at, auto piece) __attribute__((always_inline)) {
    constexpr int I = decltype(piece)::value, L = I >> 1 & (LR - 1), HALF = I & 1;
    const uint4 raw = I < 2 * LR ? kr[L] : vr[L];
    const f16x8 v = HALF ? widen_codes8(raw.z, raw.w) : widen_codes8(raw.x, raw.y);
    if constexpr (I < 2 * LR) {
      const int row = krow + L * KSTEP;
      *reinterpret_cast<f16x8*>(at + row * KB + ((kplace(kch + HALF) ^ kkey(row)) << 4)) = v;
    } else {
      const int row = vrow + L * 64;
      *reinterpret_cast<f16x8*>(at + 64 * KB + row * VB + (((fq + 4 * HALF) ^ (row & 7)) << 4)) = v;
    }
  };
  auto stage_all = [&](unsigned char* at) __attribute__((always_inline)) {
    static_for<0, 4 * LR>([&](auto i) { stage(at, i); });
  };
  const int my_row = (l16 >> 2) * 16 + (l16 & 3);           // row of K of score tile 0 (tile j: 4 j further, the same key)
  const int kbase = my_row * KB, kx = kkey(my_row);
  const int vbase = 64 * KB + l16 * VB, vx = l16 & 7;      // (row of V^T: 16 d + l16, the same key for all d)

  if (k0 < k1) load(k0);
  f16x8 qf[2][NS];
  float fac[2];
  int pos[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const uint32_t r = wrow + n * 16 + l16 < rows ? wrow + n * 16 + l16 : rows - 1;
    const int qi = (int)a.by_group.of(r), g = (int)(r - qi * a.group);
    pos[n] = q.first + qi;
    const uint16_t* p = a.Q + (q.row0 + qi) * a.ldq + ((int64_t)hk * a.group + g) * DH + fq * 8;
    fac[n] = fabsf(a.scale2) * load_queries<T, NS, 32>(p, qf[n], a.scale2 < 0.0f);
  }
  auto take_steps = [&]() {      // of the pages just staged
    seen = seen_next;
    ks = seen ? ks_next : 0.0f;
    vs = seen ? fmaxf(vs_next, kSmallStep) : 1.0f;
  };
  if (k0 < k1) {
    stage_all(lds);
    take_steps();
    load(k0 + 64);
  }
  int cur = 0;
  for (int unit = k0; unit < k1; unit += 64, cur ^= 1) {
    __syncthreads();
    const unsigned char* kv = lds + cur * STAGE;
    const bool work = unit < wend, now_seen = seen;
    const float kst = ks;
    float vst = vs;
    f32x4 sc[4][2];
    unsigned char* next = lds + (cur ^ 1) * STAGE;
    if (work) {
      // the scores, 2 k32 steps' fragments ahead; between their products the next stage is widened (behind the last step
      // that is done with what the registers hold: nobody reads it)
      f16x8 kf[2][4];
      auto read_k = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          kf[i & 1][j] = *reinterpret_cast<const f16x8*>(kv + kbase + j * 4 * KB + ((kplace(i * 4 + fq) ^ kx) << 4));
      };
      __builtin_amdgcn_s_setprio(1);      // (the wave that feeds the matrix cores goes first: 1.5 %)
      read_k(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[j][0] = sc[j][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      static_for<0, NS>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i + 1 < NS) read_k(i + 1);
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, 4>([&](auto jc) {
          constexpr int j = decltype(jc)::value, at = i * 4 + j;      // 4 NS places for 4 LR pieces, NS = 2 LR
          sc[j][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i & 1][j], qf[0][i], sc[j][0], 0, 0, 0);
          sc[j][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i & 1][j], qf[1][i], sc[j][1], 0, 0, 0);
          if constexpr ((at & 1) == 0) stage(next, std::integral_constant<int, at / 2>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      __builtin_amdgcn_s_setprio(0);
    } else {
      stage_all(next);
    }
    // (not in a branch: registers that meet behind one are copied, and a copy waits for the loads just issued.  Behind the last
    // key the last page's codes come again and are never seen)
    take_steps();
    load(unit + 128);
    if (!work) continue;
    if (unit + 64 > wfull || unit + 64 > wend || __any(!now_seen)) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int limit = now_seen ? (pos[n] < k1 - 1 ? pos[n] : k1 - 1) - (unit + fq * 16) : -1;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e >> 2][n][e & 3] = e <= limit ? sc[e >> 2][n][e & 3] : -INFINITY;
      }
      // (a page behind the last key may never have been written: an infinite step would make a NaN of the masked scores)
      if (unit + fq * 16 >= k1) vst = 1.0f;
    }
    const float lg = __builtin_amdgcn_logf(vst), rv = __builtin_amdgcn_rcpf(vst);
    float f[2], mx[2], own[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      f[n] = fmaxf(fac[n] * kst, 1e-37f);       // (zero times a masked product would not be -inf)
      mx[n] = sc[0][n][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx[n] = fmaxf(mx[n], sc[e >> 2][n][e & 3]);
      own[n] = mx[n] == -INFINITY ? mx[n] : __builtin_fmaf(mx[n], f[n], lg);
      mx[n] = column_max(own[n]);
    }
    float per = rv;
    if (__any(mx[0] > ref[0] + kRaise || mx[1] > ref[1] + kRaise || lg < quiet)) {
      const float lg_top = column_max(own[0] != -INFINITY || own[1] != -INFINITY ? lg : -INFINITY);
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (mx[n] > ref[n] + kRaise) {
          const float next = mx[n] - kTop, alpha = exp2_fast(ref[n] - next);
          l_run[n] = lower_sum(l_run[n], ref[n] - next);
          ref[n] = next;
          quiet = fmaxf(quiet, lg_top - kNear);
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[d][n] *= alpha;
        }
      if (lg < quiet && (own[0] < ref[0] - kLow || own[1] < ref[1] - kLow)) {
        per = 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float less = ref[n] != -INFINITY ? -ref[n] : 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) l_run[n] += exp2_fast(__builtin_fmaf(sc[e >> 2][n][e & 3], f[n], less));
        }
      }
    }
    float off[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) off[n] = ref[n] != -INFINITY ? lg - ref[n] : 0.0f;
    // half of the keys after the other: the weights of the second half are formed between the products of the first
    f16x8 pf[2][2], vf[4];
    auto read_v = [&](int at) __attribute__((always_inline)) {
      const int d = at % ND, u = at / ND;
      vf[at & 3] = *reinterpret_cast<const f16x8*>(kv + vbase + d * 16 * VB + (((fq + 4 * u) ^ vx) << 4));
    };
    auto weigh = [&](auto uc, auto ec) __attribute__((always_inline)) {
      constexpr int u = decltype(uc)::value, e = decltype(ec)::value;
#pragma unroll
      for (int n = 0; n < 2; ++n)
        pf[u][n][e] = (_Float16)exp2_fast(__builtin_fmaf(sc[2 * u + (e >> 2)][n][e & 3], f[n], off[n]));
    };
#pragma unroll
    for (int at = 0; at < 4; ++at) read_v(at);
    static_for<0, 8>([&](auto ec) { weigh(std::integral_constant<int, 0>{}, ec); });
    static_for<0, 2 * ND>([&](auto ac) {
      constexpr int at = decltype(ac)::value, d = at % ND, u = at / ND, E = 8 / ND;
      acc[d][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[at & 3], pf[u][0], acc[d][0], 0, 0, 0);
      acc[d][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[at & 3], pf[u][1], acc[d][1], 0, 0, 0);
      if constexpr (at + 4 < 2 * ND) read_v(at + 4);
      if constexpr (u == 0)
        static_for<0, E>([&](auto ec) { weigh(std::integral_constant<int, 1>{}, std::integral_constant<int, d * E + decltype(ec)::value>{}); });
      __builtin_amdgcn_sched_barrier(0);
    });
#pragma unroll
    for (int n = 0; n < 2; ++n) l_run[n] = __builtin_fmaf(add_weights(pf[1][n], add_weights(pf[0][n], 0.0f)), per, l_run[n]);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    float l = l_run[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const uint32_t r = wrow + n * 16 + l16;
    if (r >= rows) continue;
    const uint32_t qi = a.by_group.of(r);
    const int64_t token = q.row0 + qi, head = (int64_t)hk * a.group + (r - qi * a.group);
    if (a.n_splits > 1) {
      const int64_t at = (token * a.n_heads + head) * a.n_splits + split;
      if (fq == 0) a.ml[at] = make_float2(ref[n], l);
#pragma unroll
      for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(a.acc + at * DH + d * 16 + fq * 4) = acc[d][n];
      continue;
    }
    const float inv = ref[n] == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t* to = a.Out + token * a.ldo + head * DH + fq * 4;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      uint16_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = T::from_float(acc[d][n][e] * inv);
      *reinterpret_cast<uint2*>(to + d * 16) = make_uint2((uint32_t)w[0] | (uint32_t)w[1] << 16, (uint32_t)w[2] | (uint32_t)w[3] << 16);
    }
  }
#endif
}

// Number of splits that the tile of a row has written (see the kernels).
__device__ __forceinline__ int written_splits(const KvAttnDev& a, const KvSeq& q, int qi, int head, uint32_t tile_rows) {
  const uint32_t rows = (uint32_t)q.n_new * a.group;
  uint32_t last_row = ((uint32_t)qi * a.group + (uint32_t)head % (uint32_t)a.group) / tile_rows * tile_rows + tile_rows - 1;
  if (last_row > rows - 1) last_row = rows - 1;
  const int last = q.first + (int)a.by_group.of(last_row);
  const int end = last + 1 < q.len ? last + 1 : q.len;
  return end <= 0 ? 0 : (end + a.chunk - 1) / a.chunk;
}

// The splits of a row, up to 64 of them: sums joined with the largest of their references, a wave a row.  Bound by latency: 5
// splits of 32 rows 3.8 us.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_join_few_kernel(KvAttnDev a, uint32_t tile_rows) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef float vec __attribute__((ext_vector_type(DH / 64)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = blockIdx.z, head = blockIdx.y * 4 + wave, qi = blockIdx.x;
  const KvSeq q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  if (qi >= q.n_new || head >= a.n_heads) return;
  const int n = written_splits(a, q, qi, head, tile_rows);
  const int64_t at = ((q.row0 + qi) * a.n_heads + head) * a.n_splits;
  const float2 p = lane < n ? a.ml[at + lane] : make_float2(-INFINITY, 0.0f);
  float m = p.x;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  const float f = p.x == -INFINITY ? 0.0f : exp2_fast(p.x - m);
  float l = lower_sum(p.y, p.x - m, f);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off, 64);
  vec o = {};
  for (int i = 0; i < n; i += 8) {       // (lanes from n on have factors of zero)
    vec v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const vec*>(a.acc + (at + (i + k < n ? i + k : n - 1)) * DH + lane * (DH / 64));
#pragma unroll
    for (int k = 0; k < 8; ++k) o += v[k] * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), i + k));
  }
  const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* to = a.Out + (q.row0 + qi) * a.ldo + (int64_t)head * DH + lane * (DH / 64);
  if constexpr (DH == 128)
    *reinterpret_cast<uint32_t*>(to) = (uint32_t)T::from_float(o[0] * inv) | (uint32_t)T::from_float(o[1] * inv) << 16;
  else *to = T::from_float(o[0] * inv);
#endif
}

// More of them (few rows then).  A block has one row; DH / 4 lanes read the sums of a split, 1024 / DH splits side by side.  103
// splits of 28 rows of 128 4.8 us (a wave a row, as above, 30 for 256 splits).
[[maybe_unused]] constexpr int kMaxSplits = 1024;
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnDev a, uint32_t tile_rows) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = DH / 4, SIDE = 256 / LPR;
  __shared__ __attribute__((aligned(16))) float4 sum[SIDE][LPR];
  __shared__ float factor[kMaxSplits], red[2][4];
  const int tid = threadIdx.x, side = tid / LPR, d = tid % LPR, wave = tid >> 6;
  const int s = blockIdx.z, head = blockIdx.y, qi = blockIdx.x;
  const KvSeq q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  if (qi >= q.n_new) return;
  const int n = written_splits(a, q, qi, head, tile_rows);
  const int64_t at = ((q.row0 + qi) * a.n_heads + head) * a.n_splits;
  float2 p[kMaxSplits / 256];
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int k = 0; k < kMaxSplits / 256; ++k) {
    p[k] = k * 256 + tid < n ? a.ml[at + k * 256 + tid] : make_float2(-INFINITY, 0.0f);
    m = fmaxf(m, p[k].x);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if ((tid & 63) == 0) red[0][wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
#pragma unroll
  for (int k = 0; k < kMaxSplits / 256; ++k) {
    const float f = p[k].x == -INFINITY ? 0.0f : exp2_fast(p[k].x - m);
    if (k * 256 + tid < n) factor[k * 256 + tid] = f;
    l += lower_sum(p[k].y, p[k].x - m, f);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off, 64);
  if ((tid & 63) == 0) red[1][wave] = l;
  __syncthreads();
  l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int i = side; i < n; i += SIDE) {
    const float f = factor[i];
    const float4 v = *reinterpret_cast<const float4*>(a.acc + (at + i) * DH + d * 4);
    o.x = __builtin_fmaf(v.x, f, o.x); o.y = __builtin_fmaf(v.y, f, o.y);
    o.z = __builtin_fmaf(v.z, f, o.z); o.w = __builtin_fmaf(v.w, f, o.w);
  }
  sum[side][d] = o;
  __syncthreads();
  if (side) return;
#pragma unroll
  for (int i = 1; i < SIDE; ++i) {
    const float4 v = sum[i][d];
    o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
  }
  const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
  *reinterpret_cast<uint2*>(a.Out + (q.row0 + qi) * a.ldo + (int64_t)head * DH + d * 4) =
      make_uint2((uint32_t)T::from_float(o.x * inv) | (uint32_t)T::from_float(o.y * inv) << 16,
                 (uint32_t)T::from_float(o.z * inv) | (uint32_t)T::from_float(o.w * inv) << 16);
#endif
}

// Tiles of 16 rows times pairs of sequence and key head times 256 keys up to which the few kernel is taken, also for more than 16
// rows: it has eight times as many, shorter blocks, which decides until they fill the chip several times; then reading the
// keys again for each 16 rows does.  us few and prompt, by that number (heads of 128): 32 rows x 16 pairs x 5000 keys (640) 19
// 27, x 64 x 2000 (1024) 22 28, x 64 x 5000 (2560) 36 34; 56 x 6 x 5000 (480) 15 28, x 16 x 5000 (1280) 23 29, x 64 x 2000 (2048) 26 31,
// x 16 x 16,000 (4032) 48 41; 128 x 1 x 16,000 (504) 18 30, x 16 x 2000 (1024) 22 30, x 16 x 5000 (2560) 36 33; 256 x 4 x 5000 (1280)
// 22 30, x 64 x 500 (2048) 22 20; whole prompts 300 x 8 pairs (304) 13.1 13.4, 600 x 4 (456) 14 21, 1000 x 1 (252) 11 30, 2400 x 1 (1500) 24
// 30, 100 x 32 with four rows a token (800) 11.9 11.0.
constexpr int64_t kFewWork = 1536;

namespace {
struct KvPlan { bool prompt; int rows, tiles, n_splits, chunk; size_t acc_at, bytes; };
KvPlan kv_plan(int64_t n_tok, int n_heads, const tlq_kv_batch& b, const tlq_kv_cache& c) {
  KvPlan p;
  const int group = n_heads / c.n_kv_heads;
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  const int64_t room = (int64_t)b.max_pages * c.page, keys = b.max_len < room ? b.max_len : room;
  p.prompt = most * group > 16 && ceil_div(most * group, 16) * c.n_kv_heads * b.n_seq * ceil_div(keys, 256) > kFewWork;
  p.rows = p.prompt ? 128 : 16;
  p.tiles = (int)ceil_div(most * group, p.rows);
  const int64_t base = (int64_t)p.tiles * c.n_kv_heads * b.n_seq;
  // Split until there are about two blocks a CU, into parts of 256 keys at least.  Beyond two blocks a CU a second round of them
  // and the joining cost more than their evenness gives (us unsplit, for 256, 512 and 1024 blocks: single tokens, 131,072 keys x 4
  // key heads - 35 32 35, 8 x 4096 x 32 44 44 45 47, 32 x 1024 x 8 18 18 20 22, 64 x 8192 x 8 160 160 159 171; 64 tokens behind
  // 16,320 x 4 477 50 44 44, 4 x 100 behind 3900 x 8 122 79 61 75).
  // With the tiles of 128 rows a split costs: for 64 keys 1.6 us, with two blocks a CU 2.2, and the joined sums' way to memory
  // and back, at 4 TB/s behind another launch's 4 us.  The least by that, against parts of 512 and of 256 keys (us): 128 rows x 4
  // pairs x 16,000 keys 33 28, 256 x 6 x 16,000 38 41, x 32 x 2000 37 32, 400 x 10 x 5000 44 38, 600-token prompts x 32 heads 22
  // (unsplit) 36.
  const int64_t units = ceil_div(keys, 256);
  int64_t splits = 511 / base;
  if (splits > units) splits = units;
  if (splits < 1) splits = 1;
  if (p.prompt) {
    double least = 0.0;
    const int64_t most_splits = splits;
    for (int64_t n = splits = 1; n <= most_splits; ++n) {
      const int64_t part = ceil_div(units, n), parts = ceil_div(units, part);
      const double joined = (double)n_tok * n_heads * (double)parts * c.head_dim * 8.0 / 4e6;
      const double us = (double)part * 4.0 * (base * parts > 256 ? 2.2 : 1.6) + (parts > 1 ? 4.0 + joined : 0.0);
      if (n == 1 || us < least) { least = us; splits = n; }
    }
  }
  p.chunk = (int)(ceil_div(units, splits) * 256);
  p.n_splits = (int)ceil_div(keys, p.chunk);
  p.acc_at = align_up((size_t)n_tok * n_heads * p.n_splits * sizeof(float2), 256);
  p.bytes = p.n_splits > 1 ? p.acc_at + align_up((size_t)n_tok * n_heads * p.n_splits * c.head_dim * sizeof(float), 256) : 0;
  return p;
}
}  // namespace

size_t kv_attention_workspace(int64_t n_tok, int n_heads, const tlq_kv_batch& b, const tlq_kv_cache& c) {
  return kv_plan(n_tok, n_heads, b, c).bytes;
}

hipError_t launch_kv_attention(const void* Q, int64_t ldq, int64_t n_tok, int n_heads, float scale, const tlq_kv_batch& b,
                               const tlq_kv_cache& c, bool bf16, void* Out, int64_t ldo, void* workspace, hipStream_t stream) {
  const KvPlan p = kv_plan(n_tok, n_heads, b, c);
  KvAttnDev a{};
  a.Q = (const uint16_t*)Q; a.ldq = ldq; a.n_tok = n_tok; a.n_heads = n_heads; a.group = n_heads / c.n_kv_heads;
  a.scale2 = scale * 1.4426950408889634f;
  a.b = b; a.c = c; a.page_bits = __builtin_ctz((unsigned)c.page);
  a.Out = (uint16_t*)Out; a.ldo = ldo; a.n_splits = p.n_splits; a.chunk = p.chunk;
  a.ml = (float2*)workspace; a.acc = (float*)((unsigned char*)workspace + p.acc_at);
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  a.tiles = p.tiles;
  a.by_group = kv_div((uint32_t)a.group);
  a.by_heads = kv_div((uint32_t)c.n_kv_heads);
  const int64_t n_pairs = (int64_t)b.n_seq * c.n_kv_heads, work = (int64_t)p.tiles * p.n_splits;
  a.n_pairs = (uint32_t)n_pairs;
  a.by_work = kv_div((uint32_t)work);
  a.own_blocks = (uint32_t)(n_pairs / 8 * work);
  // (an XCD has 64 blocks at a time: more pairs than fill them only push each other's keys out of its cache, fewer leave the
  // longest tiles of the last to the end.  us with eight pairs always and by this rule: 2 x 4800 x 40 heads 600 547, 9600 x 40 1452
  // 1031; one pair always and by this rule: 16 x 1200 x 40 398 377, 4 x 2400 x 40 359 346.  Pairs that are no eight, all on XCDs of
  // their own and dealt out: 9600 x 9 heads with two rows a token 740 585, 256 tokens of two rows behind 15,744 x 9 112 68,
  // 1200 x 25 56 58)
  for (a.together_bits = 0; a.together_bits < 3 && (16 << a.together_bits) <= n_pairs && work << a.together_bits < 64; ++a.together_bits) {}
  const int64_t blocks = 8 * ((int64_t)a.own_blocks + ceil_div(n_pairs % 8 * work, 8));
  const int64_t gx = blocks < (1 << 20) ? blocks : (1 << 20);
  const dim3 grid = p.prompt ? dim3((unsigned)gx, (unsigned)ceil_div(blocks, gx))
                             : dim3((unsigned)work, (unsigned)c.n_kv_heads, (unsigned)b.n_seq);
  auto pick = [&](auto t, auto dh) {
    using T = decltype(t);
    constexpr int DH = decltype(dh)::value;
    {
      ProfScope ps("kv_attention", stream, 4.0 * (double)n_tok * n_heads * c.head_dim * (double)b.max_len);
      if (p.prompt) kv_prompt_kernel<T, DH><<<grid, 256, 0, stream>>>(a);
      else kv_few_kernel<T, DH><<<grid, 256, 0, stream>>>(a);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.n_splits == 1) return e;
    ProfScope ps("kv_join", stream, 4.0 * (double)n_tok * n_heads * p.n_splits * c.head_dim);
    if (p.n_splits <= 64)
      kv_join_few_kernel<T, DH><<<dim3((unsigned)most, (unsigned)ceil_div(n_heads, 4), (unsigned)b.n_seq), 256, 0, stream>>>(a, (uint32_t)p.rows);
    else kv_join_kernel<T, DH><<<dim3((unsigned)most, (unsigned)n_heads, (unsigned)b.n_seq), 256, 0, stream>>>(a, (uint32_t)p.rows);
    return hipGetLastError();
  };
  using W128 = std::integral_constant<int, 128>;
  using W64 = std::integral_constant<int, 64>;
  if (c.head_dim == 128) return bf16 ? pick(BF16{}, W128{}) : pick(F16{}, W128{});
  return bf16 ? pick(BF16{}, W64{}) : pick(F16{}, W64{});
}

}  // namespace tlq
