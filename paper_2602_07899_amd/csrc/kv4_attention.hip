// Causal attention over a 4-bit cache in pages.
//
// Mathematics.  Key and value of token j are codes of four bits times steps of eight significant bits, one for each 32 channels:
// products that halves hold exactly, so both matrix products run on fp16 matrix instructions with operands that are what the
// cache stands for.  With z_j = scale * log2(e) * (q . key_j) and any reference m,  out = sum_j 2^(z_j - m) value_j / sum_j 2^(z_j - m).
// m, the row's reference, is 7 below the largest z when it is set, and is set again where a lane's 8 or 16 weights come to 2^15, so that
// weights stay below that and, as normal halves, go down to 2^-29 of it, and sums are rescaled a few times a row; no maximum is
// looked for as long as the sum, which is needed anyhow, stays below (a row without a reference has one so low that every weight
// overflows; prompts set the first from their first 64 scores).  2^(z - m) is one fused product and an exponential, exact where m is
// not, so that m's rounding cancels as long as it is small.  From |m| = 2^24 on it is not, neighbouring floats being whole binary
// orders apart: such a row's scores are rounded to floats first (kFar), and the largest has the weight that m gives it.  The
// weights are rounded to halves for the second product, and the denominator sums what was rounded, in 32 bits: where one key has
// nearly all of the weight its rounding cancels.  bf16 queries are multiplied with the power of two that brings the largest of the row to
// [2^14, 2^15).  The products are transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane owns one query column and P stays in
// registers; values are stored channel by channel so that V^T's rows are read as they lie.
#include "kv4.h"
#include "kv_attention.h"

namespace tlq {

struct Kv4AttnDev : KvAttnDev { Kv4Dev d; };      // (of c the sizes)

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float kFull = 32768.0f;      // weights of a lane that call for another reference (the largest is 2^11 at least then)
constexpr float kUnset = -3.40282347e38f;      // (no score is as low, see score_factor)
__device__ __forceinline__ float ref_of(float ref) { return ref == kUnset ? -INFINITY : ref; }      // for those who join
constexpr float kFar = 16777216.0f;
// What a row's products are multiplied with.  Not zero: zero times a masked product would not be -inf.  A product of queries (2^16)
// and keys (2^16) is below 2^39, so that with 2^88 at most every score is a float.  That changes no result: two products that differ at
// all lie 2^-48 apart at least, times 2^88 all of the weight either way.
__device__ __forceinline__ float score_factor(float f) { return __builtin_amdgcn_fmed3f(f, 1e-37f, 0x1p88f); }
// The reference that a row's largest product gives; from kFar on that of the score as a float (fused, it could come out a float below)
__device__ __forceinline__ float reference(float product, float fac) {
#pragma clang fp contract(off)
  const float ref = __builtin_fmaf(product, fac, -kTop), score = product * fac;
  return fabsf(ref) >= kFar ? score - kTop : ref;
}
// keeps what a wave's lanes write for each other in LDS in order
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ uint32_t twice(uint16_t h) { return (uint32_t)h | (uint32_t)h << 16; }
// Of pair p of a lane's 16 keys, the halves of those below n
__device__ __forceinline__ uint32_t keys_below(int p, int n) {
  return (2 * p < n ? 0xffffu : 0u) | (2 * p + 1 < n ? 0xffff0000u : 0u);
}
#endif

// The 16 rows of a tile (a query and head each: the heads that share a key head are rows side by side) against one split of
// the keys.  Four waves take 64 keys each in turn and meet in LDS at the end; keys and values go from memory to registers,
// where they are widened: no barrier in the loop, the next 64 keys in flight while these are worked on.  Only their steps pass
// through the wave's own piece of LDS: a lane needs 16 of each group of channels, which sixteen lanes share; loaded by each they take
// ten more loads and 36 registers (which cost the third wave a SIMD), us that way and this: 64 x 2000 keys x 32 heads 115 99, 64 x 4096 -
// 8192 x 8 110 105, 131,072 x 4 29.3 27.8; heads of 64 64 67.  Bound by the bytes of the cache where there are many, 64 x 4096 - 8192 x 8
// 104 us, 4.4 TB/s (a copy reaches 4.8), by latency else, 1200 x 32 6.2 and 3.6 for joining five splits.  Not better: keys and values
// both two turns ahead (109 -> 121), up to 767, 1023 or 2100 blocks in place of 511.
template <typename T, int DH>
__global__ __launch_bounds__(256, 3) void kv4_few_kernel(Kv4AttnDev a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NS = DH / 32, ND = DH / 16, NG = DH / kKv4Group;      // k32 steps of a score = words of a lane's key, channel tiles, groups
  constexpr int RS = DH + 4;
  typedef uint32_t words __attribute__((ext_vector_type(NS)));
  __shared__ __attribute__((aligned(16))) float part[4][16][RS];
  __shared__ __attribute__((aligned(16))) uint16_t steps[4][2][64 * NG];      // of a wave's 64 keys: [key][group], [16 keys][group][key]
  __shared__ float2 ml[4][16];
  __shared__ float far_fac[4][16];      // 1, or of rows from kFar on the factor that their scores have before the exponent's product
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
  float fac = fabsf(a.scale2) * load_queries<T, NS, 8>(
      a.Q + (q.row0 + qi) * a.ldq + ((int64_t)hk * a.group + g) * DH + fq * (DH / 4), qf, a.scale2 < 0.0f);
  fac = score_factor(fac);
  far_fac[wave][l16] = 1.0f;
  bool far = false;                         // whether a row of the wave has such scores

  f32x4 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref = kUnset, l_run = 0.0f;         // the row's reference, this lane's share of its sum
  const Kv4Bits bits = kv4_bits();
  const int full = q.first + (int)a.by_group.of(first_row) + 1;      // keys that all rows of the tile see

  typedef uint16_t halves __attribute__((ext_vector_type(NG)));
  words kr[4];
  uint2 vr[ND];
  halves ksr, vsr;                      // steps of key fq * 16 + l16; of NG of the 16 keys, of one group
  bool seen = false;                    // this lane's 16 keys lie in a page that there is
  // The table's entries are fetched a turn before the pages they name (keys behind the last are never seen: any entry will
  // do); an entry outside the pool becomes the first page, in reach and never seen
  const int32_t* row_table = a.b.table + (int64_t)s * a.b.ld_table;
  const uint32_t n_pages = (uint32_t)a.c.n_pages;
  const int kgroup = (l16 >> 2) * 16, vgroup = fq * 16;
  uint32_t kid = 0, vid = 0;
  auto entry = [&](int key) { return (uint32_t)row_table[(key < k1 ? key : k1 - 1) >> a.page_bits]; };
  auto load_k = [&](int unit) {
    const int64_t token = ((int64_t)(kid < n_pages ? kid : 0) * a.c.n_kv_heads + hk) * a.c.page + ((unit + kgroup) & (a.c.page - 1)) + (l16 & 3);
    const uint32_t* p = a.d.k + token * (DH / 8) + fq * NS;
#pragma unroll
    for (int j = 0; j < 4; ++j) kr[j] = *reinterpret_cast<const words*>(p + j * 4 * (DH / 8));
    kid = entry(unit + 256 + kgroup);
  };
  auto load_v = [&](int unit) {
    seen = vid < n_pages;
    const int64_t slot = (int64_t)(seen ? vid : 0) * a.c.n_kv_heads + hk;
    const int at = (unit + vgroup) & (a.c.page - 1);
    const uint32_t* p = a.d.v + ((slot * DH + l16) * a.c.page + at) / 8;
    ksr = *reinterpret_cast<const halves*>(a.d.k_step + (slot * a.c.page + at + l16) * NG);
    vsr = *reinterpret_cast<const halves*>(a.d.v_step + (slot * NG + l16 / (16 / NG)) * a.c.page + at + l16 % (16 / NG) * NG);
#pragma unroll
    for (int d = 0; d < ND; ++d) vr[d] = *reinterpret_cast<const uint2*>(p + d * 2 * a.c.page);
    vid = entry(unit + 256 + vgroup);
  };

  int unit = k0 + wave * 64;
  if (unit < k1) {
    kid = entry(unit + kgroup);
    vid = entry(unit + vgroup);
    load_k(unit);
    load_v(unit);
  }
  const uint16_t* my_ks = steps[wave][0] + (kgroup + (l16 & 3)) * NG + fq * NG / 4;
  const uint16_t* my_vs = steps[wave][1] + fq * 16 * NG;
  for (; unit < k1; unit += 256) {
    // the steps of the wave's keys pass through LDS, where each lane picks those of its own
    *reinterpret_cast<halves*>(steps[wave][0] + lane * NG) = ksr;
    *reinterpret_cast<halves*>(steps[wave][1] + lane * NG) = vsr;
    wave_order();
    uint16_t ks[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) ks[j] = my_ks[j * 4 * NG];
    f32x4 sc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      const uint32_t st = twice(ks[j]);
#pragma unroll
      for (int i = 0; i < NS; ++i)
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kv4_values(kr[j][i], bits, st, st, st, st)), qf[i], sc[j], 0, 0, 0);
    }
    if (unit + 256 < k1) load_k(unit + 256);
    // lane: keys unit + 16 fq + 4 j + r of its query
    const bool hidden = unit + 64 > k1 || __any(!seen);      // keys that no row of the tile sees
    if (hidden || unit + 64 > full) {
      const int limit = seen ? (pos < k1 - 1 ? pos : k1 - 1) - (unit + fq * 16) : -1;    // last visible of the 16
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e >> 2][e & 3] = e <= limit ? sc[e >> 2][e & 3] : -INFINITY;
    }
    if (__builtin_expect(far, 0)) {
      const float f = far_fac[wave][l16];
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[j] *= f;
    }
    f16x8 pf[2];
    auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = (_Float16)exp2_of(__builtin_fmaf(sc[e >> 2][e & 3], fac, -ref));
      return add_weights(pf[1], add_weights(pf[0], 0.0f));
    };
    float sum = weigh();
    if (__any(!(sum < kFull))) {
      float mx = sc[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e >> 2][e & 3]);
      mx = column_max(mx);
      bool far_now = false;
      if (column_max(sum) >= kFull) {      // (the row's own sums: what the others hold has no part in it)
        const float next = reference(mx, fac), alpha = exp2_of(ref - next);       // (0 at the first visible key)
        l_run *= alpha;
        ref = next;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] *= alpha;
        far_now = fabsf(next) >= kFar;
      }
      if (__any(far_now)) {
        const float f = far_now ? fac : 1.0f;      // (one in a row that has been far before)
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[j] *= f;
        far_fac[wave][l16] *= f;
        wave_order();
        fac = far_now ? 1.0f : fac;
        far = true;
      }
      sum = weigh();
    }
    l_run += sum;
    uint4 vs[NG][2];
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) vs[i][u] = *reinterpret_cast<const uint4*>(my_vs + i * 16 + u * 8);
    // (steps behind the last token, or of a page that is not this sequence's, may be anything)
    if (hidden) {
      const int n = seen ? k1 - (unit + fq * 16) : 0;
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          vs[i][u].x &= keys_below(4 * u, n);
          vs[i][u].y &= keys_below(4 * u + 1, n);
          vs[i][u].z &= keys_below(4 * u + 2, n);
          vs[i][u].w &= keys_below(4 * u + 3, n);
        }
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint4 st = vs[d / 2][u];
        acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            __builtin_bit_cast(f16x8, kv4_values(u ? vr[d].y : vr[d].x, bits, st.x, st.y, st.z, st.w)), pf[u], acc[d], 0, 0, 0);
      }
    wave_order();      // (before the next turn's steps overwrite these)
    if (unit + 256 < k1) load_v(unit + 256);
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  ref = ref_of(ref);
  if (fq == 0) ml[wave][l16] = make_float2(ref, l_run);
  __syncthreads();
  const float top = fmaxf(fmaxf(ml[0][l16].x, ml[1][l16].x), fmaxf(ml[2][l16].x, ml[3][l16].x));
  const float mine = ref == -INFINITY ? 0.0f : exp2_of(ref - top);
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
  for (int w = 0; w < 4; ++w) l += ml[w][r].y * (ml[w][r].x == -INFINITY ? 0.0f : exp2_of(ml[w][r].x - m));      // (NaN stays)
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
// the next into the stage that nobody reads (one barrier a step).  All row tiles of a sequence and key head run on one XCD, the
// longest first, as far as the pairs can be dealt out evenly.  Tiles are counted from the last row, so that the one that is not
// full is the one with the fewest keys: 16 x 1200 tokens x 40 heads 366 -> 354 us, 1000 behind 1000 others x 32 433 -> 414, 4 x 2400
// 254 -> 251, 16 x 200 40 -> 42.
//   Bound by the waits of two waves a SIMD for each other, for LDS and at the barrier.  9600 tokens x 40 heads 1038 us, 910
// TFLOP/s where a large library product of halves reaches 1180; 16 x up to 1200 x 40 346, 620 TFLOP/s, since a block has 10 steps on average
// there, the diagonal's half of them idle for half of its waves, and begins and ends with a chain of loads and stores.  Rows of far scores cost the
// others 0.5 % (346 -> 348, with heads of 64 1.5 %).  Of a wave's time
// 29 % issues vector instructions, of the SIMDs' 26 % is matrix products.  Left out for measurement: widening 42 us, exponentials 32.
// Not better, us for 16 x 1200 x 40: a step in four phases that interleave two of them 469 against 371, values staged in the
// second product 5 % slower, 16 rows a wave and four waves a SIMD 493 against 359 (LDS is read twice as often).
template <typename T, int DH>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void kv4_prompt_kernel(Kv4AttnDev a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NS = DH / 32, ND = DH / 16, CPK = DH / 8, NG = DH / kKv4Group;   // k32 steps of a score, channel tiles, words of a key, groups
  constexpr int KB = DH * 2, VB = 128;                      // bytes of a row of K, of V^T in LDS
  constexpr int STAGE = 64 * KB + DH * VB, LR = DH / 64;    // LR: 8-byte loads of a thread for K, and for V
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  __shared__ float far_fac[4][2][16];                       // as in kv4_few_kernel
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
  const int split = (int)(which - turn * a.n_splits);
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
  const int rows = q.n_new * a.group, first_row = rows - ((int)turn + 1) * 128;      // (rows below 0: there are none)
  if (first_row <= -128) return;
  auto last_key = [&](int r) {      // number of keys that rows up to r see
    const int p = q.first + (int)a.by_group.of(r > 0 ? (uint32_t)r : 0);
    return p + 1 < q.len ? p + 1 : q.len;
  };
  const int end = last_key(first_row + 127);
  if (k0 >= end && a.n_splits > 1) return;
  const int k1 = end - k0 < a.chunk ? end : k0 + a.chunk;
  const int wrow = first_row + wave * 32;
  const int wend = wrow > -32 ? (last_key(wrow + 31) < k1 ? last_key(wrow + 31) : k1) : 0;     // keys of this wave
  const int wfull = wrow > -32 ? last_key(wrow) : 0;                                           // keys that all of its rows see

  f32x4 acc[ND][2];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d][0] = acc[d][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref[2] = {kUnset, kUnset}, l_run[2] = {0.0f, 0.0f};
  const Kv4Bits bits = kv4_bits();

  // what a thread moves: K rows tid / (CPK / 2) and further ones, 16 codes of a group; V channels 16 wave + l16 and 64 further, the 16
  // keys that it has the scores of.
  const int krow = tid / (CPK / 2), kch = tid % (CPK / 2) * 2, vrow = wave * 16 + l16;
  constexpr int KSTEP = 512 / CPK;                          // rows between a thread's loads of K
  const uint32_t head_words = (uint32_t)a.c.page * (DH / 8), page_stride = (uint32_t)a.c.n_kv_heads * head_words;
  const uint32_t head_steps = (uint32_t)a.c.page * NG, page_steps = (uint32_t)a.c.n_kv_heads * head_steps;
  const uint32_t n_pages = (uint32_t)a.c.n_pages, in_page = (uint32_t)a.c.page - 1;
  const uint32_t *kp = a.d.k + (uint64_t)hk * head_words, *vp = a.d.v + (uint64_t)hk * head_words;
  const uint16_t *ksp = a.d.k_step + (uint64_t)hk * head_steps, *vsp = a.d.v_step + (uint64_t)hk * head_steps;
  uint32_t koff[LR];                   // (a key's steps lie at a quarter of its words' offset)
#pragma unroll
  for (int i = 0; i < LR; ++i) koff[i] = ((uint32_t)(krow + i * KSTEP) & in_page) * (DH / 8) + kch;
  const uint32_t vat = (uint32_t)(fq * 16) & in_page, voff = (vrow * a.c.page + vat) / 8, vsoff = vrow / kKv4Group * a.c.page + vat;
  uint2 kr[LR], vr[LR];
  uint16_t ks[LR];
  uint4 vs[LR][2];
  bool seen = false, seen_next = false;
  auto load = [&](int unit) {
    const uint32_t at = (uint32_t)unit & in_page;
    const uint32_t mine = fq < 2 ? (fq == 0 ? ids[0] : ids[1]) : (fq == 2 ? ids[2] : ids[3]);
    seen_next = mine < n_pages;
    const uint32_t id = seen_next ? mine : 0;
#pragma unroll
    for (int i = 0; i < LR; ++i) {     // (DH = 128: a wave's rows lie in one group of 16 keys; 64: wave w has group w)
      const int g = DH == 128 ? (wave >> 1) + 2 * i : wave;
      uint32_t k = g == 0 ? ids[0] : g == 1 ? ids[1] : g == 2 ? ids[2] : ids[3];
      k = k < n_pages ? k : 0;
      kr[i] = *reinterpret_cast<const uint2*>(kp + ((uint64_t)k * page_stride + at * (DH / 8)) + koff[i]);
      ks[i] = (ksp + ((uint64_t)k * page_steps + at * NG))[koff[i] >> 2];
    }
    const uint32_t* p = vp + at / 8 + (uint64_t)id * page_stride;
    const uint16_t* st = vsp + at + (uint64_t)id * page_steps;
#pragma unroll
    for (int i = 0; i < LR; ++i) {
      vr[i] = *reinterpret_cast<const uint2*>(p + i * 8 * a.c.page + voff);
      vs[i][0] = *reinterpret_cast<const uint4*>(st + i * 2 * a.c.page + vsoff);
      vs[i][1] = *reinterpret_cast<const uint4*>(st + i * 2 * a.c.page + vsoff + 8);
    }
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
    if constexpr (I < 2 * LR) {
      const int row = krow + L * KSTEP;
      const uint32_t st = twice(ks[L]);
      *reinterpret_cast<uint4*>(at + row * KB + ((kplace(kch + HALF) ^ kkey(row)) << 4)) = kv4_values(HALF ? kr[L].y : kr[L].x, bits, st, st, st, st);
    } else {
      const int row = vrow + L * 64;
      const uint4 st = vs[L][HALF];
      *reinterpret_cast<uint4*>(at + 64 * KB + row * VB + (((fq + 4 * HALF) ^ (row & 7)) << 4)) =
          kv4_values(HALF ? vr[L].y : vr[L].x, bits, st.x, st.y, st.z, st.w);
    }
  };
  auto stage_all = [&](unsigned char* at) __attribute__((always_inline)) {
    static_for<0, 4 * LR>([&](auto i) { stage(at, i); });
  };
  // Steps behind the last token, or of a page that is not this sequence's, may be anything: those values are written again, as zeros.
  auto stage_tail = [&](unsigned char* at, int unit) __attribute__((always_inline)) {
    if (unit + 64 > k1 || __any(!seen_next)) {
      const int n = seen_next ? k1 - (unit + fq * 16) : 0;
#pragma unroll
      for (int i = 0; i < LR; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int row = vrow + i * 64;
          const uint4 st = vs[i][u];
          *reinterpret_cast<uint4*>(at + 64 * KB + row * VB + (((fq + 4 * u) ^ (row & 7)) << 4)) =
              kv4_values(u ? vr[i].y : vr[i].x, bits, st.x & keys_below(4 * u, n), st.y & keys_below(4 * u + 1, n),
                         st.z & keys_below(4 * u + 2, n), st.w & keys_below(4 * u + 3, n));
        }
    }
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
    const uint32_t r = wrow + n * 16 + l16 > 0 ? (uint32_t)(wrow + n * 16 + l16) : 0;
    const int qi = (int)a.by_group.of(r), g = (int)(r - qi * a.group);
    pos[n] = q.first + qi;
    const uint16_t* p = a.Q + (q.row0 + qi) * a.ldq + ((int64_t)hk * a.group + g) * DH + fq * 8;
    fac[n] = fabsf(a.scale2) * load_queries<T, NS, 32>(p, qf[n], a.scale2 < 0.0f);
    fac[n] = score_factor(fac[n]);
    far_fac[wave][n][l16] = 1.0f;
  }
  bool far = false;                         // whether a row of the wave has scores from kFar on
  if (k0 < k1) {
    stage_all(lds);
    stage_tail(lds, k0);
    seen = seen_next;
    load(k0 + 64);
  }
  int cur = 0;
  for (int unit = k0; unit < k1; unit += 64, cur ^= 1) {
    __syncthreads();
    const unsigned char* kv = lds + cur * STAGE;
    const bool work = unit < wend, now_seen = seen;
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
      __builtin_amdgcn_s_setprio(1);
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
    stage_tail(next, unit + 64);
    // (not in a branch: registers that meet behind one are copied, and a copy waits for the loads just issued.  Behind the last
    // key the last page's codes come again and are never seen)
    seen = seen_next;
    load(unit + 128);
    if (!work) continue;
    if (unit + 64 > wfull || unit + 64 > wend || __any(!now_seen)) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int limit = now_seen ? (pos[n] < k1 - 1 ? pos[n] : k1 - 1) - (unit + fq * 16) : -1;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e >> 2][n][e & 3] = e <= limit ? sc[e >> 2][n][e & 3] : -INFINITY;
      }
    }
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float f = far_fac[wave][n][l16];
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[j][n] *= f;
      }
    }
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
        pf[u][n][e] = (_Float16)exp2_of(__builtin_fmaf(sc[2 * u + (e >> 2)][n][e & 3], fac[n], -ref[n]));
    };
    // the weights of a half into the sums, behind another reference if they call for it
    auto take = [&](auto uc) __attribute__((always_inline)) {
      constexpr int u = decltype(uc)::value;
      float sum[2] = {add_weights(pf[u][0], 0.0f), add_weights(pf[u][1], 0.0f)};
      if (__any(!(sum[0] < kFull && sum[1] < kFull))) {
        bool far_now[2] = {false, false};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          float mx = sc[2 * u][n][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sc[2 * u + (e >> 2)][n][e & 3]);
          mx = column_max(mx);
          if (column_max(sum[n]) >= kFull) {      // (the row's own sums: what the others hold has no part in it)
            const float next_ref = reference(mx, fac[n]), alpha = exp2_of(ref[n] - next_ref);
            l_run[n] *= alpha;
            ref[n] = next_ref;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d][n] *= alpha;
            far_now[n] = fabsf(next_ref) >= kFar;
          }
        }
        if (__any(far_now[0] || far_now[1])) {
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float f = far_now[n] ? fac[n] : 1.0f;      // (one in a row that has been far before)
#pragma unroll
            for (int j = 2 * u; j < 4; ++j) sc[j][n] *= f;
            far_fac[wave][n][l16] *= f;
            fac[n] = far_now[n] ? 1.0f : fac[n];
          }
          wave_order();
          far = true;
        }
        static_for<0, 8>([&](auto ec) { weigh(uc, ec); });
        sum[0] = add_weights(pf[u][0], 0.0f);
        sum[1] = add_weights(pf[u][1], 0.0f);
      }
      l_run[0] += sum[0];
      l_run[1] += sum[1];
    };
    using First = std::integral_constant<int, 0>;
    using Second = std::integral_constant<int, 1>;
#pragma unroll
    for (int at = 0; at < 4; ++at) read_v(at);
    if (unit == k0) {      // the first reference, if there is a key that is not far (356 -> 353 us; the weights need no second go for it)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float mx = sc[0][n][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e >> 2][n][e & 3]);
        mx = column_max(mx) * fac[n];
        ref[n] = fabsf(mx) < kFar ? mx - kTop : kUnset;
      }
    }
    static_for<0, 8>([&](auto ec) { weigh(First{}, ec); });
    take(First{});
    static_for<0, ND>([&](auto dc) {
      constexpr int d = decltype(dc)::value, E = 8 / ND;
      acc[d][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[d & 3], pf[0][0], acc[d][0], 0, 0, 0);
      acc[d][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[d & 3], pf[0][1], acc[d][1], 0, 0, 0);
      read_v(d + 4);
      static_for<0, E>([&](auto ec) { weigh(Second{}, std::integral_constant<int, d * E + decltype(ec)::value>{}); });
      __builtin_amdgcn_sched_barrier(0);
    });
    take(Second{});
    static_for<ND, 2 * ND>([&](auto ac) {
      constexpr int at = decltype(ac)::value, d = at - ND;
      acc[d][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[at & 3], pf[1][0], acc[d][0], 0, 0, 0);
      acc[d][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[at & 3], pf[1][1], acc[d][1], 0, 0, 0);
      if constexpr (at + 4 < 2 * ND) read_v(at + 4);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  int column = l16;      // (rows are worked out again, not held in registers through the loop)
  asm volatile("" : "+v"(column));
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    float l = l_run[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    ref[n] = ref_of(ref[n]);
    if (wrow + n * 16 + column < 0) continue;
    const uint32_t r = (uint32_t)(wrow + n * 16 + column);
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

size_t kv4_attention_workspace(int64_t n_tok, int n_heads, const tlq_kv_batch& b, const tlq_kv4_cache& c) {
  return kv_plan(n_tok, n_heads, b, kv4_sizes(c), true).bytes;
}

hipError_t launch_kv4_attention(const void* Q, int64_t ldq, int64_t n_tok, int n_heads, float scale, const tlq_kv_batch& b,
                                const tlq_kv4_cache& c, bool bf16, void* Out, int64_t ldo, void* workspace, hipStream_t stream) {
  const tlq_kv_cache sizes = kv4_sizes(c);
  const KvPlan p = kv_plan(n_tok, n_heads, b, sizes, true);
  dim3 grid;
  Kv4AttnDev a;
  static_cast<KvAttnDev&>(a) = kv_attn_dev(p, Q, ldq, n_tok, n_heads, scale, b, sizes, Out, ldo, workspace, &grid);
  a.d = {c.k, c.k_step, c.v, c.v_step};
  {
    ProfScope ps(p.prompt ? "kv4_prompt" : "kv4_few", stream, 4.0 * (double)n_tok * n_heads * c.head_dim * (double)b.max_len);
    auto pick = [&](auto t, auto dh) {
      using T = decltype(t);
      constexpr int DH = decltype(dh)::value;
      if (p.prompt) kv4_prompt_kernel<T, DH><<<grid, 256, 0, stream>>>(a);
      else kv4_few_kernel<T, DH><<<grid, 256, 0, stream>>>(a);
    };
    using W128 = std::integral_constant<int, 128>;
    using W64 = std::integral_constant<int, 64>;
    if (c.head_dim == 128) bf16 ? pick(BF16{}, W128{}) : pick(F16{}, W128{});
    else bf16 ? pick(BF16{}, W64{}) : pick(F16{}, W64{});
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess || p.n_splits == 1) return e;
  return launch_kv_join(p, a, p.prompt, bf16, stream);
}

}  // namespace tlq
