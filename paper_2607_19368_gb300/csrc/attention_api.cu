// C entry points of the attention calls: argument checks, and the kernels' view
// of the caller's structures.
#include "attention.cuh"

using namespace sls;

namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;
// the kernels count cached tokens, and up to a step's or a batch of pages' more, in 32 bits
constexpr int64_t kMaxCached = ((int64_t)1 << 31) - 1024;

// The running maximum is taken of unscaled scores.
bool scale_ok(float s) { return s > 0.f && s <= 3.402823466e38f; }

bool aligned16(const void* p) { return p != nullptr && (uintptr_t)p % 16 == 0; }

// A packed-rows argument of T tokens; the pointer may be NULL when there are none.
int rows_view(const sls_rows_t* r, int64_t T, int head_dim, RowsView* out) {
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
bool packed_ok(const sls_kv_cache_t* c) { return c->batch <= SLS_MAX_PACKED_SEQUENCES; }

int cache_view(const sls_kv_cache_t* c, int q_heads, CacheView* v) {
  if (!c || q_heads < 1 || c->kv_heads < 1) return SLS_ERR_INVALID_ARG;
  if (c->batch < 0 || c->max_pages < 0 || c->num_pages < 1 || c->table_ld < c->max_pages)
    return SLS_ERR_INVALID_ARG;
  if (q_heads % c->kv_heads != 0) return SLS_ERR_INVALID_ARG;
  if (c->dtype != SLS_BF16 && c->dtype != SLS_F16) return SLS_ERR_UNSUPPORTED;
  if (c->head_dim < 8 || c->head_dim % 8 != 0 || c->head_dim > SLS_MAX_HEAD_DIM)
    return SLS_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return SLS_ERR_UNSUPPORTED;
  if (q_heads / c->kv_heads > SLS_MAX_HEAD_GROUP) return SLS_ERR_UNSUPPORTED;
  if (c->batch > kMaxTokens || c->num_pages > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > kMaxCached) return SLS_ERR_UNSUPPORTED;
  if (c->page_stride < 0 || c->page_stride % 8 || c->slot_stride % 8 || c->head_stride % 8 ||
      c->slot_stride < c->head_dim || c->head_stride < c->head_dim)
    return SLS_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v)) return SLS_ERR_INVALID_ARG;
  if (c->batch > 0 && (!c->kv_lens || (c->max_pages > 0 && !c->page_table)))
    return SLS_ERR_INVALID_ARG;
  v->k = (char*)c->k;
  v->v = (char*)c->v;
  v->page_b = c->page_stride * 2;
  v->slot_b = c->slot_stride * 2;
  v->head_b = c->head_stride * 2;
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

}  // namespace

extern "C" {

int sls_qkv_append(const sls_rows_t* q, const sls_rows_t* k, const sls_rows_t* v, int64_t T,
                   int q_heads, const sls_kv_cache_t* cache, const int32_t* cu_seqlens,
                   const int32_t* positions, const void* q_weight, const void* k_weight,
                   float eps, const sls_rope_t* rope, const sls_rows_t* q_out, void* stream) {
  AppendArgs a{};
  int st = cache_view(cache, q_heads, &a.c);
  if (st != SLS_OK) return st;
  if (T < 0 || T > kMaxTokens || !(eps >= 0.f)) return SLS_ERR_INVALID_ARG;
  if (!cu_seqlens && T != cache->batch) return SLS_ERR_INVALID_ARG;
  if (cu_seqlens && !packed_ok(cache)) return SLS_ERR_UNSUPPORTED;
  const int hd = cache->head_dim;
  if ((st = rows_view(q, T, hd, &a.q)) != SLS_OK || (st = rows_view(k, T, hd, &a.k)) != SLS_OK ||
      (st = rows_view(v, T, hd, &a.v)) != SLS_OK || (st = rows_view(q_out, T, hd, &a.out)) != SLS_OK)
    return st;
  if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight)))
    return SLS_ERR_INVALID_ARG;
  if (rope) {
    if (rope->pairs < 0 || 2 * rope->pairs > hd || (rope->pairs > 0 && !rope->inv_freq))
      return SLS_ERR_INVALID_ARG;
    a.inv_freq = rope->inv_freq;
    a.pairs = rope->pairs;
    a.interleaved = rope->interleaved != 0;
    a.rope_scale = rope->scale;
  }
  a.T = T;
  a.q_heads = q_heads;
  a.cu = cu_seqlens;
  a.positions = positions;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.eps = eps;
  return launch_qkv_append(a, cache->dtype, (cudaStream_t)stream);
}

size_t sls_attention_prefill_workspace_size(int64_t T, int q_heads, const sls_kv_cache_t* cache) {
  CacheView c;
  if (T < 0 || T > kMaxTokens || cache_view(cache, q_heads, &c) != SLS_OK) return 0;
  return attention_prefill_workspace(c, T, q_heads);
}

int sls_attention_prefill(const sls_rows_t* q, int64_t T, int q_heads,
                          const sls_kv_cache_t* cache, const int32_t* cu_seqlens, int causal,
                          float scale, const sls_rows_t* out, void* workspace,
                          size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  int st = cache_view(cache, q_heads, &a.c);
  if (st != SLS_OK) return st;
  if (T < 0 || T > kMaxTokens || !cu_seqlens || !scale_ok(scale)) return SLS_ERR_INVALID_ARG;
  if (!packed_ok(cache)) return SLS_ERR_UNSUPPORTED;
  if ((st = rows_view(q, T, cache->head_dim, &a.q)) != SLS_OK ||
      (st = rows_view(out, T, cache->head_dim, &a.out)) != SLS_OK)
    return st;
  a.T = T;
  a.q_heads = q_heads;
  a.cu = cu_seqlens;
  a.causal = causal != 0;
  a.scale = scale;
  const size_t need = attention_prefill_workspace(a.c, T, q_heads);
  if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return SLS_ERR_WORKSPACE;
  return launch_attention_prefill(a, cache->dtype, workspace, (cudaStream_t)stream);
}

size_t sls_attention_decode_workspace_size(int q_heads, const sls_kv_cache_t* cache) {
  CacheView c;
  return cache_view(cache, q_heads, &c) == SLS_OK ? attention_decode_workspace(c, q_heads) : 0;
}

int sls_attention_decode(const sls_rows_t* q, int q_heads, const sls_kv_cache_t* cache,
                         float scale, const sls_rows_t* out, void* workspace,
                         size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  int st = cache_view(cache, q_heads, &a.c);
  if (st != SLS_OK) return st;
  if (!scale_ok(scale)) return SLS_ERR_INVALID_ARG;
  a.T = cache->batch;
  if ((st = rows_view(q, a.T, cache->head_dim, &a.q)) != SLS_OK ||
      (st = rows_view(out, a.T, cache->head_dim, &a.out)) != SLS_OK)
    return st;
  a.q_heads = q_heads;
  a.scale = scale;
  const size_t need = attention_decode_workspace(a.c, q_heads);
  if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return SLS_ERR_WORKSPACE;
  return launch_attention_decode(a, cache->dtype, workspace, (cudaStream_t)stream);
}

int sls_attention_status(void* stream) {
  int* word[2] = {nullptr, nullptr};
  int st = prefill_status_word(&word[0]);
  if (st == SLS_OK) st = decode_status_word(&word[1]);
  if (st != SLS_OK) return st;
  // both are read and cleared, whatever the first one holds
  const int prefill = sls_workspace_status(word[0], stream);
  const int decode = sls_workspace_status(word[1], stream);
  return prefill != SLS_OK ? prefill : decode;
}

}  // extern "C"
