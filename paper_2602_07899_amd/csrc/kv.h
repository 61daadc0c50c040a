// What the kernels of the 8-bit cache share: a sequence of a batch, from lengths that live on the device.
#pragma once
#include "common.h"

namespace tlq {

struct KvSeq {
  int64_t row0;      // first of its new rows in the call's matrices
  int n_new;         // new rows within the host's bound, those before the sequence's first token among them
  int first;         // position of row row0 (negative: that many rows lie before the first token)
  int len;           // tokens, those beyond the table or the host's bounds left out
};
// Values that no valid batch has are held to what is addressable.
__device__ __forceinline__ KvSeq kv_sequence(const tlq_kv_batch& b, int page, int64_t n_tok, int s) {
  KvSeq q;
  int64_t r0 = b.cu_new[s], r1 = b.cu_new[s + 1];
  r0 = r0 < 0 ? 0 : (r0 > n_tok ? n_tok : r0);
  r1 = r1 < r0 ? r0 : (r1 > n_tok ? n_tok : r1);
  const int len = b.lens[s] < 0 ? 0 : b.lens[s];
  q.row0 = r0;
  const int rows = (int)(r1 - r0);
  q.n_new = rows < b.max_new ? rows : b.max_new;
  q.first = len - rows;
  const int64_t room = (int64_t)b.max_pages * page;
  q.len = q.first + q.n_new;       // (negative where all of those rows lie before the first token)
  if (q.len > b.max_len) q.len = b.max_len;
  if (q.len > room) q.len = (int)room;
  return q;
}
// The page that the table names, or -1.
__device__ __forceinline__ int kv_page(const tlq_kv_batch& b, const tlq_kv_cache& c, int s, int index) {
  const int id = b.table[(int64_t)s * b.ld_table + index];
  return id >= 0 && id < c.n_pages ? id : -1;
}

}  // namespace tlq
