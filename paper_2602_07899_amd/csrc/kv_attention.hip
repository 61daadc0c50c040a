// Causal attention over an 8-bit cache in pages.
//
// Mathematics.  Key j of a head is kcode_j * ks(j), value j is vcode_j * vs(j), with one step ks, vs for each page and head.
// With z_j = scale * log2(e) * ks(j) * (q . kcode_j) + log2(vs(j)) and any reference m,
//   out = sum_j 2^(z_j - m) vcode_j  /  sum_j 2^(z_j - m) / vs(j):
// the values' step goes into the exponent for nothing, so that the codes enter the second product as they are and the
// weights that are rounded to 16 bits are those of the contributions, not of the probabilities - a page of small values
// (a first token's) cannot push the rest below the smallest half.  m is the running maximum of z less 15: the largest
// weight is exactly 2^15, and weights stay normal halves down to 2^-29 of it (with the largest at 1, 2^-14: over 10^5 keys
// what falls below would show).  Both products run on fp16 matrix instructions whatever x_dtype is: codes are exact in
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

struct KvAttnDev {
  const uint16_t* Q; int64_t ldq, n_tok; int n_heads, group; float scale2;    // scale * log2(e)
  tlq_kv_batch b; tlq_kv_cache c; int page_bits;
  uint16_t* Out; int64_t ldo;
  int n_splits, chunk;          // keys of a split
  float2* ml; float* acc;       // per (row, head, split): reference and sum; [head_dim] sums of codes
};

#if defined(__HIP_DEVICE_COMPILE__)
constexpr float kSmallStep = 1e-30f;    // (a step of zero: its codes' page counts as zeros)
// The reference for a largest exponent m: the weight of m is 2^15 exactly.  (Exponents so large that m - 15 is not exact have
// weight 1: a rounded reference could push it beyond the largest half.)
__device__ __forceinline__ float weight_ref(float m) { return m - (fabsf(m) < 4194304.0f ? 15.0f : 0.0f); }
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
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// N queries' channels of a lane as halves; the factor that undoes their prescale.  `rows`: lanes (lane ^ 16, lane ^ 32)
// that hold the other channels of the same query.
template <typename T, int N>
__device__ __forceinline__ float load_queries(const uint16_t* p, f16x8 (&qf)[N]) {
  u16x8 raw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) raw[i] = *reinterpret_cast<const u16x8*>(p + 8 * i);
  if constexpr (std::is_same<T, F16>::value) {
#pragma unroll
    for (int i = 0; i < N; ++i) qf[i] = __builtin_bit_cast(f16x8, raw[i]);
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
  // exponent field of the largest -> 127 + 14; rows of zeros, subnormals, infinities or NaN keep factors that are finite
  int k = 141 - (int)(top >> 7);
  k = k < -112 ? -112 : (k > 126 ? 126 : k);
  const float up = __builtin_bit_cast(float, (uint32_t)(127 + k) << 23);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) qf[i][e] = (_Float16)(BF16::to_float(raw[i][e]) * up);
  return __builtin_bit_cast(float, (uint32_t)(127 - k) << 23);
}
#endif

// The 16 rows of a tile (a query and head each: the heads that share a key head are rows side by side) against one split of
// the keys.  Four waves take 64 keys each in turn and meet in LDS at the end; keys and values go from memory to registers,
// where they are widened: no LDS, no barrier in the loop, the next 64 keys in flight while these are worked on.
// For few rows, bound by the bytes of the cache.
template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void kv_few_kernel(KvAttnDev a) {
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
  const int64_t rows = (int64_t)q.n_new * a.group;
  const int64_t first_row = (int64_t)tile * 16;
  if (first_row >= rows) return;
  const int64_t row = first_row + l16 < rows ? first_row + l16 : rows - 1;
  const int qi = (int)(row / a.group), g = (int)(row % a.group);
  const int pos = q.first + qi;
  const int64_t last_row = first_row + 15 < rows ? first_row + 15 : rows - 1;
  const int last = q.first + (int)(last_row / a.group);      // the tile's latest position
  const int end = last + 1 < q.len ? last + 1 : q.len;
  const int k0 = split * a.chunk;
  if (k0 >= end && a.n_splits > 1) return;
  const int k1 = end - k0 < a.chunk ? end : k0 + a.chunk;

  f16x8 qf[NS];
  const float unscale = load_queries<T, NS>(
      a.Q + (q.row0 + qi) * a.ldq + ((int64_t)hk * a.group + g) * DH + fq * (DH / 4), qf);
  const float fac = a.scale2 * unscale;

  f32x4 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m_run = -INFINITY, ref = -INFINITY, l_run = 0.0f;      // largest exponent, its reference, this lane's share of the sum

  uint4 kr[4][LW], vr[ND];
  float ks = 0.0f, vs = 1.0f;
  bool seen = false;                    // this lane's 16 keys lie in a page that there is
  const int64_t head_bytes = (int64_t)a.c.page * DH;
  auto slot_of = [&](int key, bool& ok) {     // (a page that is not there: the pool's first, in reach and never seen)
    const int id = key < end ? kv_page(a.b, a.c, s, key >> a.page_bits) : -1;
    ok = id >= 0;
    return (int64_t)(ok ? id : 0) * a.c.n_kv_heads + hk;
  };
  auto load_k = [&](int unit) {
    bool ok;
    const int key = unit + (l16 >> 2) * 16;
    const int8_t* p = a.c.k + slot_of(key, ok) * head_bytes + (int64_t)((key & (a.c.page - 1)) + (l16 & 3)) * DH + fq * (DH / 4);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < LW; ++i) kr[j][i] = *reinterpret_cast<const uint4*>(p + j * 4 * DH + i * 16);
  };
  auto load_v = [&](int unit) {
    const int key = unit + fq * 16;
    const int64_t slot = slot_of(key, seen);
    const int8_t* p = a.c.v + slot * head_bytes + (key & (a.c.page - 1)) + (int64_t)l16 * a.c.page;
#pragma unroll
    for (int d = 0; d < ND; ++d) vr[d] = *reinterpret_cast<const uint4*>(p + (int64_t)d * 16 * a.c.page);
    ks = seen ? a.c.k_step[slot] : 0.0f;
    vs = seen ? fmaxf(a.c.v_step[slot], kSmallStep) : 1.0f;
  };

  int unit = k0 + wave * 64;
  if (unit < k1) { load_k(unit); load_v(unit); }
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
    const float f = fac * ks, lg = __log2f(vs), rv = 1.0f / vs;
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
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (mx > m_run) {
      const float next = weight_ref(mx), alpha = exp2_fast(ref - next);       // (0 at the first visible key)
      m_run = mx;
      ref = next;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= alpha;
    }
    const float from = ref == -INFINITY ? 0.0f : ref;
    f16x8 pf[2];
    float ps = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = exp2_fast(sc[j][r] - from);
        ps += e;
        pf[j >> 1][(j & 1) * 4 + r] = (_Float16)e;
      }
    l_run = __builtin_fmaf(ps, rv, l_run);
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
    if (ml[w][r].x != -INFINITY) l += ml[w][r].y * exp2_fast(ml[w][r].x - m);
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = (part[0][r][d0 + e] + part[1][r][d0 + e]) + (part[2][r][d0 + e] + part[3][r][d0 + e]);
  const int64_t orow = first_row + r, token = q.row0 + orow / a.group, head = (int64_t)hk * a.group + orow % a.group;
  if (a.n_splits > 1) {
    const int64_t at = (token * a.n_heads + head) * a.n_splits + split;
    if ((tid & 15) == 0) a.ml[at] = make_float2(m, l);
#pragma unroll
    for (int e = 0; e < PER; e += 4)
      *reinterpret_cast<float4*>(a.acc + at * DH + d0 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
    return;
  }
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
  uint16_t w[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) w[e] = T::from_float(o[e] * inv);
  uint16_t* to = a.Out + token * a.ldo + head * DH + d0;
#pragma unroll
  for (int e = 0; e < PER; e += 4)
    *reinterpret_cast<uint2*>(to + e) = make_uint2((uint32_t)w[e] | (uint32_t)w[e + 1] << 16, (uint32_t)w[e + 2] | (uint32_t)w[e + 3] << 16);
#endif
}

// The splits of a row: sums joined with the largest of their references.  A block has one row; DH / 4 lanes read the sums of a
// split, 1024 / DH splits side by side.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnDev a, int tile_rows) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = DH / 4, SIDE = 256 / LPR;
  __shared__ __attribute__((aligned(16))) float4 sum[SIDE][LPR];
  __shared__ float lsum[SIDE];
  const int tid = threadIdx.x, side = tid / LPR, d = tid % LPR;
  const int s = blockIdx.z, head = blockIdx.y, qi = blockIdx.x;
  const KvSeq q = kv_sequence(a.b, a.c.page, a.n_tok, s);
  if (qi >= q.n_new) return;
  // the splits that its tile has written (see the kernels)
  const int64_t rows = (int64_t)q.n_new * a.group;
  int64_t last_row = ((int64_t)qi * a.group + head % a.group) / tile_rows * tile_rows + tile_rows - 1;
  if (last_row > rows - 1) last_row = rows - 1;
  const int last = q.first + (int)(last_row / a.group);
  const int end = last + 1 < q.len ? last + 1 : q.len;
  const int n = end <= 0 ? 0 : (end + a.chunk - 1) / a.chunk;
  const int64_t at = ((q.row0 + qi) * a.n_heads + head) * a.n_splits;
  float m = -INFINITY;
  for (int i = 0; i < n; ++i) m = fmaxf(m, a.ml[at + i].x);
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float l = 0.0f;
  for (int i = side; i < n; i += SIDE) {
    const float2 p = a.ml[at + i];
    if (p.x == -INFINITY) continue;
    const float f = exp2_fast(p.x - m);
    const float4 v = *reinterpret_cast<const float4*>(a.acc + (at + i) * DH + d * 4);
    l += p.y * f;
    o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f;
  }
  sum[side][d] = o;
  if (d == 0) lsum[side] = l;
  __syncthreads();
  if (side) return;
  for (int i = 1; i < SIDE; ++i) {
    const float4 v = sum[i][d];
    o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
    l += lsum[i];
  }
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
  *reinterpret_cast<uint2*>(a.Out + (q.row0 + qi) * a.ldo + (int64_t)head * DH + d * 4) =
      make_uint2((uint32_t)T::from_float(o.x * inv) | (uint32_t)T::from_float(o.y * inv) << 16,
                 (uint32_t)T::from_float(o.z * inv) | (uint32_t)T::from_float(o.w * inv) << 16);
#endif
}

namespace {
struct KvPlan { int tiles, n_splits, chunk; size_t acc_at, bytes; };
KvPlan kv_plan(int64_t n_tok, int n_heads, const tlq_kv_batch& b, const tlq_kv_cache& c) {
  KvPlan p;
  const int group = n_heads / c.n_kv_heads;
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  p.tiles = (int)ceil_div(most * group, 16);
  const int64_t room = (int64_t)b.max_pages * c.page, keys = b.max_len < room ? b.max_len : room;
  const int64_t base = (int64_t)p.tiles * c.n_kv_heads * b.n_seq;
  int64_t splits = ceil_div(1024, base);
  const int64_t units = ceil_div(keys, 256);
  if (splits > units) splits = units;
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
  if ((int64_t)p.tiles * p.n_splits > 0x7fffffffLL) return hipErrorInvalidValue;
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  const dim3 grid((unsigned)(p.tiles * p.n_splits), (unsigned)c.n_kv_heads, (unsigned)b.n_seq);
  auto pick = [&](auto t, auto dh) {
    using T = decltype(t);
    constexpr int DH = decltype(dh)::value;
    {
      ProfScope ps("kv_attention", stream, 4.0 * (double)n_tok * n_heads * c.head_dim * (double)b.max_len);
      kv_few_kernel<T, DH><<<grid, 256, 0, stream>>>(a);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.n_splits == 1) return e;
    ProfScope ps("kv_join", stream, 4.0 * (double)n_tok * n_heads * p.n_splits * c.head_dim);
    kv_join_kernel<T, DH><<<dim3((unsigned)most, (unsigned)n_heads, (unsigned)b.n_seq), 256, 0, stream>>>(a, 16);
    return hipGetLastError();
  };
  using W128 = std::integral_constant<int, 128>;
  using W64 = std::integral_constant<int, 64>;
  if (c.head_dim == 128) return bf16 ? pick(BF16{}, W128{}) : pick(F16{}, W128{});
  return bf16 ? pick(BF16{}, W64{}) : pick(F16{}, W64{});
}

}  // namespace tlq
