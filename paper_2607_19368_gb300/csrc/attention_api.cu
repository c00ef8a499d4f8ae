// C entry points of the attention calls: argument checks, and the kernels' view
// of the caller's structures.
#include "attention_args.cuh"

using namespace sls;

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
