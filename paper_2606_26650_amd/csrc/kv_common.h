// Shared by the paged-cache kernels: descriptor checks, the geometry in device
// form, and the sanitised view of a batch.
#pragma once

#include "kernels.h"

namespace catq {

struct KvGeom {
  const int32_t* table;
  const int32_t* cu;
  const int32_t* ctx;
  int64_t n_tokens;
  int32_t n_q, n_kv, d;
  int32_t ps_log2, bt_log2;   // page_size, scale_block
  int32_t n_pages, max_pages;
  int32_t n_seqs, max_new;
};

// Sequence s of the batch: its first row, its rows that lie inside the token
// arrays (at most max_new), and the tokens before them.  What the device arrays
// hold is not known on the host, so it is bounded here.
struct KvSeq {
  int64_t row0;
  int32_t n, ctx;
};
__device__ __forceinline__ KvSeq kv_seq(const KvGeom& g, int s) {
  const int64_t a = g.cu[s], b = g.cu[s + 1];
  KvSeq r;
  r.row0 = a < 0 ? 0 : a;
  const int64_t end = b < g.n_tokens ? b : g.n_tokens;
  const int64_t n = a < 0 ? 0 : end - a;
  r.n = n <= 0 ? 0 : (int32_t)(n < g.max_new ? n : g.max_new);
  r.ctx = g.ctx[s];
  return r;
}
// positions a page table row can hold
__device__ __forceinline__ int64_t kv_capacity(const KvGeom& g) {
  return (int64_t)g.max_pages << g.ps_log2;
}
// element offset of token `tok` (of a page) and kv head h in either code array (the
// four-token interleave of v is inside a multiple of four tokens)
__device__ __forceinline__ int64_t kv_code_base(const KvGeom& g, int page, int h, int tok) {
  return ((((int64_t)page * g.n_kv + h) << g.ps_log2) + tok) * g.d;
}
__device__ __forceinline__ int64_t kv_scale_index(const KvGeom& g, int page, int h, int tok) {
  return (((int64_t)page * g.n_kv + h) << (g.ps_log2 - g.bt_log2)) + (tok >> g.bt_log2);
}

catq_status kv_check(const catq_kv_desc* d, const catq_kv_cache* c, const catq_kv_batch* b);
catq_status kv_check_sizes(const catq_kv_desc* d, const catq_kv_batch* b);
KvGeom kv_geom(const catq_kv_desc* d, const catq_kv_batch* b);

}  // namespace catq
