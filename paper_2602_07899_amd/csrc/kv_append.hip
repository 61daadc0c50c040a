// New keys and values into the pages of an 8-bit cache.
#include "kv.h"

namespace tlq {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

#if defined(__HIP_DEVICE_COMPILE__)
constexpr float kKvTop = 127.0f;
__device__ __forceinline__ float finite_abs(float x) { return __builtin_isfinite(x) ? fabsf(x) : 0.0f; }
__device__ __forceinline__ int kv_code(float x, float step) {
  const float q = __builtin_rintf(x / step);
  return x != x ? 0 : (int)__builtin_amdgcn_fmed3f(q, -kKvTop, kKvTop);
}
__device__ __forceinline__ int byte_of(uint32_t w, int i) { return (int)(int8_t)(w >> (8 * i)); }
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)(d & 255) << 24;
}
// the codes of one page's step: quotients by the reciprocal, and divisions where one of eight lies so near a tie that it
// could decide (error of the product at most 128 * 1.5 ulp) or the reciprocal is not a normal number
struct KvStep {
  float step, rd, lim;
  __device__ __forceinline__ explicit KvStep(float s)
      : step(s), rd(__builtin_amdgcn_rcpf(s)), lim(s < 1e36f ? 0.49999976f - 4.8e-7f * 128.0f : -1.0f) {}
  __device__ __forceinline__ void codes8(const float (&x)[8], uint32_t& lo, uint32_t& hi) const {
    float n[8], tie = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = x[e] * rd;
      n[e] = __builtin_rintf(t);
      tie = fmaxf(tie, fabsf(t - n[e]));
    }
    if (!(tie < lim)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[e] = __builtin_rintf(x[e] / step);
        asm volatile("" : "+v"(n[e])::"memory");      // (in the branch, not computed and dropped)
      }
    }
    int c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = x[e] != x[e] ? 0 : (int)__builtin_amdgcn_fmed3f(n[e], -kKvTop, kKvTop);
    lo = pack4(c[0], c[1], c[2], c[3]);
    hi = pack4(c[4], c[5], c[6], c[7]);
  }
};
#endif

// A few new tokens a sequence: a block owns one page of one head, for K (blockIdx.z = 0) or V, and nobody else writes there.
// Bound by latency: the table's entry, the rows, the step, the codes one after the other: 64 sequences x 8 heads of 128 5.9 us.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_append_few_kernel(const uint16_t* __restrict__ K, int64_t ldk, const uint16_t* __restrict__ V,
                                                        int64_t ldv, int64_t n_tok, tlq_kv_batch b, tlq_kv_cache c, int max_touch) {
  #if defined(__HIP_DEVICE_COMPILE__)
  __shared__ float red[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = (int)(blockIdx.x / (unsigned)max_touch), j = (int)(blockIdx.x % (unsigned)max_touch), h = blockIdx.y;
  const bool val = blockIdx.z != 0;
  const int page = c.page;
  const KvSeq q = kv_sequence(b, page, n_tok, s);
  const int begin = q.first < 0 ? 0 : q.first;              // position of the first token that is new
  if (begin >= q.len) return;
  const int index = begin / page + j;
  if (index > (q.len - 1) / page) return;
  const int id = kv_page(b, c, s, index);
  if (id < 0) return;
  const int p0 = index * page;
  const int lo = begin > p0 ? begin - p0 : 0, hi = q.len - p0 < page ? q.len - p0 : page;   // its new tokens
  const uint16_t* x = (val ? V : K) + (int64_t)h * DH;
  const int64_t ld = val ? ldv : ldk, r0 = q.row0 + p0 - q.first;      // (row of the page's token 0, may lie before the rows)
  const int64_t slot = (int64_t)id * c.n_kv_heads + h;
  int8_t* codes = (val ? c.v : c.k) + slot * page * DH;
  float* at = (val ? c.v_step : c.k_step) + slot;

  float m = 0.0f;
  for (int i = tid; i < (hi - lo) * (DH / 8); i += 256) {
    const u16x8 v = *reinterpret_cast<const u16x8*>(x + (r0 + lo + i / (DH / 8)) * ld + i % (DH / 8) * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(T::to_float(v[e])));
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if (lane == 0) red[wave] = m;
  const float was = lo > 0 ? *at : 0.0f;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  float step = fmaxf(m, kRangeFloor) / kKvTop;
  step = was > step ? was : step;
  if (tid == 0) *at = step;
  const float again = was / step;
  const bool redo = lo > 0 && was != step;

  if (!val) {
    const int first = redo ? 0 : lo;
    for (int i = tid; i < (hi - first) * (DH / 8); i += 256) {
      const int r = first + i / (DH / 8), d = i % (DH / 8) * 8;
      uint2* to = reinterpret_cast<uint2*>(codes + r * DH + d);
      int n[8];
      if (r < lo) {
        const uint2 o = *to;
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = (int)__builtin_rintf((float)byte_of(e < 4 ? o.x : o.y, e & 3) * again);
      } else {
        const u16x8 v = *reinterpret_cast<const u16x8*>(x + (r0 + r) * ld + d);
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = kv_code(T::to_float(v[e]), step);
      }
      *to = make_uint2(pack4(n[0], n[1], n[2], n[3]), pack4(n[4], n[5], n[6], n[7]));
    }
    return;
  }
  // V: eight tokens of one channel at a time; tokens of the eight that are not new keep their codes (or have them stored again)
  const int first = (redo ? 0 : lo) / 8, last = (hi + 7) / 8;
  for (int i = tid; i < (last - first) * DH; i += 256) {
    const int r = (first + i / DH) * 8, d = i % DH;
    uint2* to = reinterpret_cast<uint2*>(codes + d * page + r);
    uint2 o = make_uint2(0, 0);
    if (r < lo || r + 8 > hi) o = *to;
    int n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      n[e] = byte_of(e < 4 ? o.x : o.y, e & 3);
      if (r + e < lo) {
        if (redo) n[e] = (int)__builtin_rintf((float)n[e] * again);
      } else if (r + e < hi) {
        n[e] = kv_code(T::to_float(x[(r0 + r + e) * ld + d]), step);
      }
    }
    *to = make_uint2(pack4(n[0], n[1], n[2], n[3]), pack4(n[4], n[5], n[6], n[7]));
  }
#endif
}

// Many: a block owns one page of one head, K and V: the largest value of its new rows, the step, the codes; nobody else writes
// there, so no atomics on memory.  A thread has pieces of four tokens x eight channels (up to U: half of them K's, the others
// V's), which stay in registers between the maximum and the codes, so that rows are read once.  V's codes turn in LDS, where a
// piece is eight words of four tokens.  Codes of tokens that the page held before are stored again where the step has grown.
// Bound by bytes: 16 x 613 tokens x 32 heads of 128 in pages of 32 60 - 66 us, 3.7 - 4.0 TB/s (with divisions throughout, rows
// read twice and V two bytes at a time 108).
template <typename T, int DH, int U>
__global__ __launch_bounds__(256) void kv_append_kernel(const uint16_t* __restrict__ K, int64_t ldk, const uint16_t* __restrict__ V,
                                                        int64_t ldv, int64_t n_tok, tlq_kv_batch b, tlq_kv_cache c, int max_touch) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = DH / 8, MAXP = U * 4096 / DH, PITCH = MAXP / 4 + 1;      // lanes of a row, tokens of a page at most, words
  __shared__ uint32_t turn[DH * PITCH];
  __shared__ uint32_t most[2];
  const int tid = threadIdx.x;
  const int s = (int)(blockIdx.x / (unsigned)max_touch), j = (int)(blockIdx.x % (unsigned)max_touch), h = blockIdx.y;
  const int page = c.page;
  const KvSeq q = kv_sequence(b, page, n_tok, s);
  const int begin = q.first < 0 ? 0 : q.first;              // position of the first token that is new
  if (begin >= q.len) return;
  const int index = begin / page + j;
  if (index > (q.len - 1) / page) return;
  const int id = kv_page(b, c, s, index);
  if (id < 0) return;
  const int p0 = index * page;
  const int lo = begin > p0 ? begin - p0 : 0, hi = q.len - p0 < page ? q.len - p0 : page;   // its new tokens
  const int64_t r0 = q.row0 + p0 - q.first;                 // row of the page's token 0 (may lie before the rows)
  const int64_t slot = (int64_t)id * c.n_kv_heads + h;
  int8_t *kc = c.k + slot * page * DH, *vc = c.v + slot * page * DH;
  const float was[2] = {lo > 0 ? c.k_step[slot] : 0.0f, lo > 0 ? c.v_step[slot] : 0.0f};

  if (tid < 2) most[tid] = 0;
  const int half = (page >> 2) * LPR;                        // pieces of K, and of V
  u16x8 x[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 256 + tid, v = i >= half, k = v ? i - half : i;
    const int t = k / LPR * 4, d = k % LPR * 8;
    const uint16_t* p = (v ? V : K) + (int64_t)h * DH + d;
    const int64_t ld = v ? ldv : ldk;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[u][e] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (k < half && t + e >= lo && t + e < hi) x[u][e] = *reinterpret_cast<const u16x8*>(p + (r0 + t + e) * ld);
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int f = 0; f < 8; ++f) m = fmaxf(m, finite_abs(T::to_float(x[u][e][f])));
#pragma unroll
    for (int off = 4; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));      // (eight lanes have pieces of one of the two)
    const int v = u * 256 + tid >= half;
    if ((tid & 7) == 0) atomicMax(&most[v], __builtin_bit_cast(uint32_t, m));       // (not negative: ordered as integers)
  }
  __syncthreads();
  float step[2], again[2];
  bool redo[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    step[v] = fmaxf(__builtin_bit_cast(float, most[v]), kRangeFloor) / kKvTop;
    step[v] = was[v] > step[v] ? was[v] : step[v];
    again[v] = was[v] / step[v];
    redo[v] = lo > 0 && was[v] != step[v];
  }
  if (tid == 0) {
    c.k_step[slot] = step[0];
    c.v_step[slot] = step[1];
  }
  const KvStep sk(step[0]), sv(step[1]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 256 + tid, v = i >= half, k = v ? i - half : i;
    const int t = k / LPR * 4, d = k % LPR * 8;
    if (k >= half || t + 4 <= lo || t >= hi) continue;
    uint32_t a[4], z[4];
    const KvStep& st = v ? sv : sk;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f[8];
#pragma unroll
      for (int g = 0; g < 8; ++g) f[g] = T::to_float(x[u][e][g]);
      st.codes8(f, a[e], z[e]);
    }
    if (!v) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e >= lo && t + e < hi) *reinterpret_cast<uint2*>(kc + (t + e) * DH + d) = make_uint2(a[e], z[e]);
    } else {
      // four rows of eight bytes -> eight words of four tokens
      auto words = [&](const uint32_t (&w)[4], int first) {
        const uint32_t p = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), r = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
        const uint32_t y = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), m = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
        uint32_t* to = turn + (d + first) * PITCH + (t >> 2);
        to[0] = __builtin_amdgcn_perm(r, p, 0x05040100u);
        to[PITCH] = __builtin_amdgcn_perm(r, p, 0x07060302u);
        to[2 * PITCH] = __builtin_amdgcn_perm(m, y, 0x05040100u);
        to[3 * PITCH] = __builtin_amdgcn_perm(m, y, 0x07060302u);
      };
      words(a, 0);
      words(z, 4);
    }
  }
  auto scaled_again = [](uint32_t w, float f) {
    int n[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) n[e] = (int)__builtin_rintf((float)byte_of(w, e) * f);
    return pack4(n[0], n[1], n[2], n[3]);
  };
  if (redo[0])
    for (int i = tid; i < lo * (DH / 8); i += 256) {
      uint2* to = reinterpret_cast<uint2*>(kc) + i;
      const uint2 o = *to;
      *to = make_uint2(scaled_again(o.x, again[0]), scaled_again(o.y, again[0]));
    }
  __syncthreads();
  // V: 16 tokens of one channel at a time; those of the 16 that are not new keep their codes (or have them stored again)
  const int first = (redo[1] ? 0 : lo) / 16, count = (hi + 15) / 16 - first;
  for (int i = tid; i < count * DH; i += 256) {
    const int d = i / count, t = (first + i % count) * 16;
    uint4* to = reinterpret_cast<uint4*>(vc + d * page + t);
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = turn[d * PITCH + (t >> 2) + e];
    if (t < lo || t + 16 > hi) {
      const uint4 old = *to;
      const uint32_t o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t before = redo[1] ? scaled_again(o[e], again[1]) : o[e];
        uint32_t r = 0;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int at = t + e * 4 + f;
          r |= (at < lo ? before : at < hi ? w[e] : o[e]) & (0xffu << (8 * f));
        }
        w[e] = r;
      }
    }
    *to = make_uint4(w[0], w[1], w[2], w[3]);
  }
#endif
}

int64_t kv_append_pages(int64_t n_tok, const tlq_kv_batch& b, const tlq_kv_cache& c) {
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  return (most - 1 + c.page - 1) / c.page + 1;
}

hipError_t launch_kv_append(const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch& b,
                            const tlq_kv_cache& c, bool bf16, hipStream_t stream) {
  ProfScope ps("kv_append", stream, 6.0 * (double)n_tok * c.n_kv_heads * c.head_dim);
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  const int max_touch = (int)kv_append_pages(n_tok, b, c);
  const int64_t gx = (int64_t)b.n_seq * max_touch;
  // Where less than half a page is new the pieces of the other kernel are mostly empty; pages of 256 x 128 would need twice the
  // registers there are for two blocks.  64 sequences x 8 heads of 128, us few and many, by new tokens: pages of 16, 8 7.9 8.2, 16
  // 9.1 8.5; of 64, 1 5.7 12.4, 24 13.0 14.0, 32 14.6 13.9, 128 28.9 21.8; of 128, 32 16.2 21.1, 64 26.4 25.7; of 256, 128 47 66,
  // 256 87 89; 16 x 613 x 32 heads, pages of 16 104 74, 32 91 53, 128 121 78, 256 142 161
  const bool few = 2 * most < c.page || c.page * c.head_dim > 16384;
  const dim3 grid((unsigned)gx, (unsigned)c.n_kv_heads, few ? 2 : 1);
  auto go = [&](auto kern) {
    kern<<<grid, 256, 0, stream>>>((const uint16_t*)K, ldk, (const uint16_t*)V, ldv, n_tok, b, c, max_touch);
  };
  auto pick = [&](auto t) {
    using T = decltype(t);
    const int pieces = c.page * c.head_dim / 16;       // of K and V
    if (few) c.head_dim == 128 ? go(kv_append_few_kernel<T, 128>) : go(kv_append_few_kernel<T, 64>);
    else if (c.head_dim == 128) {
      if (pieces <= 256) go(kv_append_kernel<T, 128, 1>);
      else if (pieces <= 512) go(kv_append_kernel<T, 128, 2>);
      else go(kv_append_kernel<T, 128, 4>);
    } else {
      if (pieces <= 256) go(kv_append_kernel<T, 64, 1>);
      else if (pieces <= 512) go(kv_append_kernel<T, 64, 2>);
      else go(kv_append_kernel<T, 64, 4>);
    }
  };
  bf16 ? pick(BF16{}) : pick(F16{});
  return hipGetLastError();
}

}  // namespace tlq
