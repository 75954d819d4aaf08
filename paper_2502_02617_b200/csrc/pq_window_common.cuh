// The paged window's layout: pool [page][kv head][K | V][token of the page][head_dim] (see include/polarquant.h).
#pragma once

#include "pq_common.cuh"

namespace pq {

// Element of the pool where row `slot` of (page, kv head, K or V) starts.
__device__ __forceinline__ int64_t window_row(const Paging& pg, int n_kv_heads, int d, int page, int h, int kv, int slot) {
  return ((((int64_t)page * n_kv_heads + h) * 2 + kv) * pg.page_tokens + slot) * d;
}

inline bool window_head_dim(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

inline int32_t window_paging_from(const pq_paging* p, Paging* out) {
  if (p == nullptr || p->page_table_dev == nullptr) return PQ_ERR_INVALID_ARG;
  if (p->page_tokens <= 0 || p->page_tokens % 16 || p->pages_per_seq <= 0 || p->n_pages <= 0) return PQ_ERR_INVALID_ARG;
  // a warp's next step, up to 64 tokens behind the last one it reads, is a position in 32 bits too
  if ((int64_t)p->page_tokens * p->pages_per_seq > (1ll << 31) - 256) return PQ_ERR_UNSUPPORTED;
  if ((uintptr_t)p->page_table_dev & 3) return PQ_ERR_ALIGNMENT;
  out->table = p->page_table_dev; out->page_tokens = p->page_tokens; out->pages_per_seq = p->pages_per_seq;
  out->n_pages = p->n_pages;
  return PQ_OK;
}

}  // namespace pq
