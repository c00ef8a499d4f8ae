// C entry points of the calls that make the cache smaller: argument checks, and the kernels'
// view of the caller's structures.
#include "attention_args.cuh"
#include "cache8.cuh"

using namespace sls;

namespace {

bool dtype_ok(int dtype) { return dtype == SLS_BF16 || dtype == SLS_F16; }

// with_v: values' scales are wanted too
int scale_view(const sls_kv_scales_t* s, const CacheView& c, bool with_v, ScaleView* v) {
  if (!s || !s->k || (with_v && !s->v)) return SLS_ERR_INVALID_ARG;
  if ((uintptr_t)s->k % 4 || (uintptr_t)s->v % 4) return SLS_ERR_INVALID_ARG;
  if (s->block != 16 && s->block != 32 && s->block != 64 && s->block != 128)
    return SLS_ERR_UNSUPPORTED;
  if (s->block > (1 << c.page_shift)) return SLS_ERR_UNSUPPORTED;
  if (s->page_stride < 1 || s->block_stride < 1 || s->head_stride < 1) return SLS_ERR_INVALID_ARG;
  v->k = s->k;
  v->v = s->v;
  v->page = s->page_stride;
  v->block = s->block_stride;
  v->head = s->head_stride;
  v->shift = 4;
  while ((1 << v->shift) < s->block) ++v->shift;
  return SLS_OK;
}

int code_cache(const sls_kv_cache_t* cache, const sls_kv_scales_t* scales, int q_heads, int dtype,
               CacheView* c, ScaleView* s) {
  const int st = cache_view(cache, q_heads, c, 1);
  if (st != SLS_OK) return st;
  if (!dtype_ok(dtype)) return SLS_ERR_UNSUPPORTED;
  return scale_view(scales, *c, true, s);
}

// A cache of codes (scales given) or of 16-bit elements; keys alone where values are not read.
int any_cache(const sls_kv_cache_t* cache, const sls_kv_scales_t* scales, int q_heads,
              bool keys_only, CacheView* c, ScaleView* s) {
  if (!cache) return SLS_ERR_INVALID_ARG;
  sls_kv_cache_t own = *cache;
  if (keys_only) own.v = own.k;
  const int st = cache_view(&own, q_heads, c, scales ? 1 : 2);
  if (st != SLS_OK || !scales) return st;
  return scale_view(scales, *c, !keys_only, s);
}

int weight_view(const sls_kv_weights_t* w, const CacheView& c, WeightView* v) {
  if (!w || !aligned16(w->data)) return SLS_ERR_INVALID_ARG;
  if (w->page_stride < 0 || w->page_stride % 4 || w->head_stride % 4 ||
      w->head_stride < (1 << c.page_shift))
    return SLS_ERR_INVALID_ARG;
  // every page has weights of its own
  if (c.num_pages > 1 && w->page_stride < (1 << c.page_shift)) return SLS_ERR_INVALID_ARG;
  v->data = w->data;
  v->page = w->page_stride;
  v->head = w->head_stride;
  return SLS_OK;
}

}  // namespace

extern "C" {

int sls_qkv_append_q8(const sls_rows_t* q, const sls_rows_t* k, const sls_rows_t* v, int64_t T,
                      int q_heads, const sls_kv_cache_t* cache, const sls_kv_scales_t* scales,
                      int dtype, const int32_t* cu_seqlens, const int32_t* positions,
                      const void* q_weight, const void* k_weight, float eps,
                      const sls_rope_t* rope, const sls_rows_t* q_out, void* stream) {
  AppendArgs a{};
  ScaleView s{};
  int st = code_cache(cache, scales, q_heads, dtype, &a.c, &s);
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
  return launch_qkv_append_q8(a, s, cache->dtype, dtype, (cudaStream_t)stream);
}

size_t sls_attention_prefill_q8_workspace_size(int64_t T, int q_heads,
                                               const sls_kv_cache_t* cache,
                                               const sls_kv_scales_t* scales, int dtype) {
  CacheView c;
  ScaleView s;
  if (T < 0 || T > kMaxTokens || code_cache(cache, scales, q_heads, dtype, &c, &s) != SLS_OK)
    return 0;
  const ExpandPlan p = cache_expand_plan(c);
  return p.table_b + 2 * p.pool_b + attention_prefill_workspace(c, T, q_heads);
}

int sls_attention_prefill_q8(const sls_rows_t* q, int64_t T, int q_heads,
                             const sls_kv_cache_t* cache, const sls_kv_scales_t* scales,
                             int dtype, const int32_t* cu_seqlens, int causal, float scale,
                             const sls_rows_t* out, void* workspace, size_t workspace_bytes,
                             void* stream) {
  AttnArgs a{};
  ScaleView s{};
  int st = code_cache(cache, scales, q_heads, dtype, &a.c, &s);
  if (st != SLS_OK) return st;
  if (T < 0 || T > kMaxTokens || !cu_seqlens || !scale_ok(scale)) return SLS_ERR_INVALID_ARG;
  if (!packed_ok(cache)) return SLS_ERR_UNSUPPORTED;
  if ((st = rows_view(q, T, cache->head_dim, &a.q)) != SLS_OK ||
      (st = rows_view(out, T, cache->head_dim, &a.out)) != SLS_OK)
    return st;
  if (T == 0 || cache->batch == 0) return SLS_OK;
  a.T = T;
  a.q_heads = q_heads;
  a.cu = cu_seqlens;
  a.causal = causal != 0;
  a.scale = scale;
  const ExpandPlan p = cache_expand_plan(a.c);
  const size_t pages = p.table_b + 2 * p.pool_b;
  const size_t need = pages + attention_prefill_workspace(a.c, T, q_heads);
  if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return SLS_ERR_WORKSPACE;
  const CacheView codes = a.c;
  st = launch_cache_expand(codes, s, cache->dtype, dtype, p, workspace, &a.c, (cudaStream_t)stream);
  if (st != SLS_OK) return st;
  return launch_attention_prefill(a, dtype, (char*)workspace + pages, (cudaStream_t)stream);
}

size_t sls_attention_decode_q8_workspace_size(int q_heads, const sls_kv_cache_t* cache,
                                              const sls_kv_scales_t* scales, int dtype) {
  CacheView c;
  ScaleView s;
  return code_cache(cache, scales, q_heads, dtype, &c, &s) == SLS_OK
             ? attention_decode_q8_workspace(c, q_heads)
             : 0;
}

int sls_attention_decode_q8(const sls_rows_t* q, int q_heads, const sls_kv_cache_t* cache,
                            const sls_kv_scales_t* scales, int dtype, float scale,
                            const sls_rows_t* out, void* workspace, size_t workspace_bytes,
                            void* stream) {
  AttnArgs a{};
  ScaleView s{};
  int st = code_cache(cache, scales, q_heads, dtype, &a.c, &s);
  if (st != SLS_OK) return st;
  if (!scale_ok(scale)) return SLS_ERR_INVALID_ARG;
  a.T = cache->batch;
  if ((st = rows_view(q, a.T, cache->head_dim, &a.q)) != SLS_OK ||
      (st = rows_view(out, a.T, cache->head_dim, &a.out)) != SLS_OK)
    return st;
  a.q_heads = q_heads;
  a.scale = scale;
  const size_t need = attention_decode_q8_workspace(a.c, q_heads);
  if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return SLS_ERR_WORKSPACE;
  return launch_attention_decode_q8(a, s, cache->dtype, dtype, workspace, (cudaStream_t)stream);
}

size_t sls_attention_weights_workspace_size(int64_t T, int q_heads, const sls_kv_cache_t* cache,
                                            const sls_kv_scales_t* scales, int dtype) {
  CacheView c;
  ScaleView s;
  if (T < 0 || T > kMaxTokens || !dtype_ok(dtype) ||
      any_cache(cache, scales, q_heads, true, &c, &s) != SLS_OK)
    return 0;
  return attention_weights_workspace(c, T, q_heads);
}

int sls_attention_weights(const sls_rows_t* q, int64_t T, int q_heads,
                          const sls_kv_cache_t* cache, const sls_kv_scales_t* scales, int dtype,
                          const int32_t* cu_seqlens, int causal, float scale,
                          const sls_kv_weights_t* weights, void* workspace,
                          size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  ScaleView s{};
  WeightView w{};
  int st = any_cache(cache, scales, q_heads, true, &a.c, &s);
  if (st != SLS_OK) return st;
  if (!dtype_ok(dtype) || (!scales && cache->dtype != dtype)) return SLS_ERR_UNSUPPORTED;
  if ((st = weight_view(weights, a.c, &w)) != SLS_OK) return st;
  if (T < 0 || T > kMaxTokens || !scale_ok(scale)) return SLS_ERR_INVALID_ARG;
  if (!cu_seqlens && T != cache->batch) return SLS_ERR_INVALID_ARG;
  if (cu_seqlens && !packed_ok(cache)) return SLS_ERR_UNSUPPORTED;
  if ((st = rows_view(q, T, cache->head_dim, &a.q)) != SLS_OK) return st;
  a.T = T;
  a.q_heads = q_heads;
  a.cu = cu_seqlens;
  a.causal = causal != 0;
  a.scale = scale;
  const size_t need = attention_weights_workspace(a.c, T, q_heads);
  if (need > 0 && (!aligned16(workspace) || workspace_bytes < need)) return SLS_ERR_WORKSPACE;
  return launch_attention_weights(a, s, w, cache->dtype, dtype, workspace, (cudaStream_t)stream);
}

int sls_cache_evict(const sls_kv_cache_t* cache, const sls_kv_scales_t* scales,
                    const sls_kv_weights_t* weights, int64_t keep, int64_t first, int64_t last,
                    int32_t* kept, int32_t* kv_lens, void* stream) {
  EvictArgs a{};
  if (!cache) return SLS_ERR_INVALID_ARG;
  int st = any_cache(cache, scales, cache->kv_heads, false, &a.c, &a.s);
  if (st != SLS_OK) return st;
  if ((st = weight_view(weights, a.c, &a.w)) != SLS_OK) return st;
  if (keep < 0 || first < 0 || last < 0 || keep > 0x7fffffff || first > keep || last > keep - first)
    return SLS_ERR_INVALID_ARG;
  if (cache->batch > 0 && (kv_lens != cache->kv_lens || (keep > 0 && !kept)))
    return SLS_ERR_INVALID_ARG;
  a.keep = (int)keep;
  a.first = (int)first;
  a.last = (int)last;
  a.kept = kept;
  a.lens = kv_lens;
  return launch_cache_evict(a, cache->dtype, (cudaStream_t)stream);
}

}  // extern "C"
