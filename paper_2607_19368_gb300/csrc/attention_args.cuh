// Argument checks that the attention and cache calls share: the kernels' view of the
// caller's structures.
#pragma once

#include "attention.cuh"

namespace sls {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;
// the kernels count cached tokens, and up to a step's or a batch of pages' more, in 32 bits
constexpr int64_t kMaxCached = ((int64_t)1 << 31) - 1024;

// The running maximum is taken of unscaled scores.
inline bool scale_ok(float s) { return s > 0.f && s <= 3.402823466e38f; }

inline bool aligned16(const void* p) { return p != nullptr && (uintptr_t)p % 16 == 0; }

// A packed-rows argument of T tokens; the pointer may be NULL when there are none.
inline int rows_view(const sls_rows_t* r, int64_t T, int head_dim, RowsView* out) {
  if (!r) return SLS_ERR_INVALID_ARG;
  if (T > 0 && !aligned16(r->data)) return SLS_ERR_INVALID_ARG;
  if (r->token_stride % 8 != 0 || r->head_stride % 8 != 0) return SLS_ERR_INVALID_ARG;
  if (r->token_stride < 0 || r->head_stride < 0) return SLS_ERR_INVALID_ARG;
  if (head_dim > 0 && r->head_stride < head_dim) return SLS_ERR_INVALID_ARG;
  out->data = (char*)r->data;
  out->token_b = r->token_stride * 2;
  out->head_b = r->head_stride * 2;
  return SLS_OK;
}

// Packed calls look a token's or an item's sequence up among all of them, while other warps
// wait: 134 us an item in prefill of 16384 short sequences, and some 50 passes over the
// lengths at most, by estimate 0.1 s of the second that a wait lasts at 65536.
inline bool packed_ok(const sls_kv_cache_t* c) { return c->batch <= SLS_MAX_PACKED_SEQUENCES; }

// element: bytes of an element, 2 or 1 (caches of 8-bit codes).
inline int cache_view(const sls_kv_cache_t* c, int q_heads, CacheView* v, int element = 2) {
  const bool wide = element == 2;
  const int step = 16 / element;  // elements of 16 bytes
  if (!c || q_heads < 1 || c->kv_heads < 1) return SLS_ERR_INVALID_ARG;
  if (c->batch < 0 || c->max_pages < 0 || c->num_pages < 1 || c->table_ld < c->max_pages)
    return SLS_ERR_INVALID_ARG;
  if (q_heads % c->kv_heads != 0) return SLS_ERR_INVALID_ARG;
  if (wide ? c->dtype != SLS_BF16 && c->dtype != SLS_F16
           : c->dtype != SLS_I8 && c->dtype != SLS_E4M3)
    return SLS_ERR_UNSUPPORTED;
  if (c->head_dim < step || c->head_dim % step != 0 || c->head_dim > SLS_MAX_HEAD_DIM)
    return SLS_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return SLS_ERR_UNSUPPORTED;
  if (q_heads / c->kv_heads > SLS_MAX_HEAD_GROUP) return SLS_ERR_UNSUPPORTED;
  if (c->batch > kMaxTokens || c->num_pages > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > kMaxCached) return SLS_ERR_UNSUPPORTED;
  if (c->page_stride < 0 || c->page_stride % step || c->slot_stride % step ||
      c->head_stride % step ||
      c->slot_stride < c->head_dim || c->head_stride < c->head_dim)
    return SLS_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v)) return SLS_ERR_INVALID_ARG;
  if (c->batch > 0 && (!c->kv_lens || (c->max_pages > 0 && !c->page_table)))
    return SLS_ERR_INVALID_ARG;
  v->k = (char*)c->k;
  v->v = (char*)c->v;
  v->page_b = c->page_stride * element;
  v->slot_b = c->slot_stride * element;
  v->head_b = c->head_stride * element;
  v->num_pages = c->num_pages;
  v->page_shift = 0;
  while ((1 << v->page_shift) < c->page_size) ++v->page_shift;
  v->kv_heads = c->kv_heads;
  v->head_dim = c->head_dim;
  v->table = c->page_table;
  v->table_ld = c->table_ld;
  v->max_pages = c->max_pages;
  v->kv_lens = c->kv_lens;
  v->B = (int)c->batch;
  return SLS_OK;
}

}  // namespace sls
