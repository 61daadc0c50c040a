// New keys and values into the pages of an 8-bit cache.
#include "kv.h"

namespace tlq {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

constexpr float kKvTop = 127.0f;
__device__ __forceinline__ float finite_abs(float x) { return __builtin_isfinite(x) ? fabsf(x) : 0.0f; }
__device__ __forceinline__ int kv_code(float x, float step) {
  const float q = __builtin_rintf(x / step);
  return x != x ? 0 : (int)__builtin_amdgcn_fmed3f(q, -kKvTop, kKvTop);
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)(d & 255) << 24;
}
__device__ __forceinline__ int byte_of(uint32_t w, int i) { return (int)(int8_t)(w >> (8 * i)); }

// A block owns one page of one head, for K (blockIdx.z = 0) or V: the largest value of its new rows, the step, the codes;
// nobody else writes there, so no atomics.  Codes of tokens that the page held before are stored again where the step has
// grown.  Bound by bytes for prompts, by latency for single tokens.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_append_kernel(const uint16_t* __restrict__ K, int64_t ldk, const uint16_t* __restrict__ V,
                                                        int64_t ldv, int64_t n_tok, tlq_kv_batch b, tlq_kv_cache c, int max_touch) {
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
}

hipError_t launch_kv_append(const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch& b,
                            const tlq_kv_cache& c, bool bf16, hipStream_t stream) {
  ProfScope ps("kv_append", stream, 6.0 * (double)n_tok * c.n_kv_heads * c.head_dim);
  const int64_t most = b.max_new < n_tok ? b.max_new : n_tok;
  const int max_touch = (int)((most - 1 + c.page - 1) / c.page + 1);     // pages that `most` tokens can lie in
  const int64_t gx = (int64_t)b.n_seq * max_touch;
  if (gx > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, (unsigned)c.n_kv_heads, 2);
  auto go = [&](auto kern) {
    kern<<<grid, 256, 0, stream>>>((const uint16_t*)K, ldk, (const uint16_t*)V, ldv, n_tok, b, c, max_touch);
  };
  if (c.head_dim == 128) bf16 ? go(kv_append_kernel<BF16, 128>) : go(kv_append_kernel<F16, 128>);
  else bf16 ? go(kv_append_kernel<BF16, 64>) : go(kv_append_kernel<F16, 64>);
  return hipGetLastError();
}

}  // namespace tlq
