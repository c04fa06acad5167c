// The caller's paged key-value pools as the kernels see them (hsd_kv_append, hsd_paged_attention).
#pragma once
#include "common.cuh"

namespace hsd {

struct PoolView {
  unsigned char *k, *v;
  long long head_bytes, page_bytes, token_bytes;
  int n_pages, page;
};

// Lists of 32-bit numbers stand where they can be read as such.
static inline bool words(const void *a, const void *b, const void *c = nullptr) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c)) & 3) == 0;
}

// What both calls ask of a pool: 16-byte pieces of rows of head_dim values, sizes that 32-bit positions can name.
static inline int pool_view(const hsd_kv_pool *p, int n_kv_heads, int head_dim, int pages_per_seq, PoolView &v) {
  if (!p || !p->k || !p->v || p->n_pages <= 0 || p->page_size <= 0 || pages_per_seq <= 0 || n_kv_heads <= 0) return HSD_E_INVALID_ARG;
  if (p->dtype != HSD_F32 && p->dtype != HSD_BF16) return HSD_E_INVALID_ARG;
  if (p->head_stride < 0 || p->page_stride < 0 || p->token_stride < 0) return HSD_E_INVALID_ARG;
  const int e = p->dtype == HSD_F32 ? 4 : 2;
  v.k = static_cast<unsigned char *>(p->k);
  v.v = static_cast<unsigned char *>(p->v);
  v.head_bytes = p->head_stride * e;
  v.page_bytes = p->page_stride * e;
  v.token_bytes = p->token_stride * e;
  if (((reinterpret_cast<uintptr_t>(p->k) | reinterpret_cast<uintptr_t>(p->v)) & 15) || ((v.head_bytes | v.page_bytes | v.token_bytes) & 15)) return HSD_E_INVALID_ARG;
  if (head_dim != 32 && head_dim != 64 && head_dim != 128) return HSD_E_UNSUPPORTED;
  if ((long long)pages_per_seq * p->page_size > 0x7FFFFF00ll) return HSD_E_TOO_LARGE;
  v.n_pages = p->n_pages;
  v.page = p->page_size;
  return HSD_OK;
}

}  // namespace hsd
