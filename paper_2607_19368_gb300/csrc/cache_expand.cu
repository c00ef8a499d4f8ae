// The pages of a batch's sequences written out in 16 bits, code times scale: what the prefill
// kernel reads in place of a cache of codes.
//
// The products are exact where the scale is a power of two (a code has at most 8 significant
// bits, as bfloat16 has), so nothing is lost against codes multiplied in the attention kernel;
// that would convert every key and value once for each of its query tiles, on the CUDA cores
// that its softmax is short of.  A copy, bound by memory: one byte read and two written an
// element, once, then found in L2 for prompts of up to some 30k tokens of 8 heads.  8192 tokens of 8
// heads of 128: 10.5 us (4.8 TB/s), of 491 for the whole call.
//
// Keys and values of a page lie by head, each head's slots one after the other.
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int CE_T = 256;

// Two products rounded; float16 cut to +-65504, NaN kept.
template <typename E>
SLS_DEV uint32_t ce_narrow(float x, float y) {
  const uint32_t u = Half2<E>::narrow(x, y);
  if constexpr (std::is_same<E, __half>::value) {
    const __half2 most = __half2half2(__ushort_as_half(0x7bff)), h = *reinterpret_cast<const __half2*>(&u);
    const __half2 cut = __hmax2_nan(__hmin2_nan(h, most), __hneg2(most));
    return *reinterpret_cast<const uint32_t*>(&cut);
  }
  return u;
}

// grid: (sequence and page of its table, 2 x key heads)
template <typename E, typename C>
__global__ void __launch_bounds__(CE_T)
cache_expand_kernel(const __grid_constant__ CacheView c, const __grid_constant__ ScaleView s,
                    bool compact, int32_t* table, char* pool, size_t pool_b) {
  const int seq = blockIdx.x / c.max_pages, col = blockIdx.x - seq * c.max_pages;
  const bool keys = (int)blockIdx.y < c.kv_heads;
  const int h = keys ? blockIdx.y : blockIdx.y - c.kv_heads;
  at_go();
  at_wait_ahead();
  const int64_t len = cache_len(c, seq);
  const int used = (int)min((int64_t)1 << c.page_shift, len - ((int64_t)col << c.page_shift));
  if (used <= 0) return;
  const int64_t page = c.table[seq * c.table_ld + col];
  const bool real = page >= 0 && page < c.num_pages;
  const int64_t to = compact ? (int64_t)seq * c.max_pages + col : page;
  if (compact && blockIdx.y == 0 && threadIdx.x == 0) table[to] = real ? (int)to : -1;
  if (!real) return;
  const unsigned vecs = c.head_dim >> 4;  // of 16 codes
  const char* src = (keys ? c.k : c.v) + page * c.page_b + h * c.head_b;
  const float* sc = (keys ? s.k : s.v) + page * s.page + h * s.head;
  E* dst = reinterpret_cast<E*>(pool + (keys ? 0 : pool_b)) +
           (((to * c.kv_heads + h) << c.page_shift) * c.head_dim);
#pragma unroll 1
  for (unsigned i = threadIdx.x; i < used * vecs; i += CE_T) {
    const int slot = i / vecs, v = i - slot * vecs;
    float x[16];
    codes_float<C>(*reinterpret_cast<const uint4*>(src + slot * c.slot_b + 16 * v), x);
    const float f = sc[(slot >> s.shift) * s.block];
    uint32_t y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = ce_narrow<E>(x[2 * e] * f, x[2 * e + 1] * f);
    uint4* d = reinterpret_cast<uint4*>(dst + (int64_t)slot * c.head_dim + 16 * v);
    d[0] = make_uint4(y[0], y[1], y[2], y[3]);
    d[1] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

template <typename E>
int launch(const CacheView& c, const ScaleView& s, int code, const ExpandPlan& p, int32_t* table,
           char* pool, cudaStream_t stream) {
  const dim3 grid((unsigned)(c.B * (int64_t)c.max_pages), (unsigned)(2 * c.kv_heads));
  return code == SLS_I8
             ? at_launch(cache_expand_kernel<E, I8>, grid, CE_T, 0, 1, stream, c, s, p.compact,
                         table, pool, p.pool_b)
             : at_launch(cache_expand_kernel<E, E4M3>, grid, CE_T, 0, 1, stream, c, s, p.compact,
                         table, pool, p.pool_b);
}

}  // namespace

ExpandPlan cache_expand_plan(const CacheView& c) {
  ExpandPlan p;
  const int64_t table = (int64_t)c.B * c.max_pages;
  p.compact = table <= c.num_pages;
  p.pages = p.compact ? table : c.num_pages;
  p.table_b = p.compact ? sls_align256((size_t)table * 4) : 0;
  p.pool_b = sls_align256(((size_t)p.pages * c.kv_heads * c.head_dim << c.page_shift) * 2);
  return p;
}

int launch_cache_expand(const CacheView& c, const ScaleView& s, int code, int dtype,
                        const ExpandPlan& p, void* workspace, CacheView* out,
                        cudaStream_t stream) {
  char* pool = (char*)workspace + p.table_b;
  int32_t* table = p.compact ? (int32_t*)workspace : nullptr;
  *out = c;
  out->k = pool;
  out->v = pool + p.pool_b;
  out->slot_b = (int64_t)c.head_dim * 2;
  out->head_b = out->slot_b << c.page_shift;
  out->page_b = out->head_b * c.kv_heads;
  out->num_pages = p.pages > 0 ? p.pages : 1;
  if (p.compact) out->table = table, out->table_ld = c.max_pages;
  if (c.B == 0 || c.max_pages == 0) return SLS_OK;
  if ((int64_t)c.B * c.max_pages > 0x7fffffff || 2 * c.kv_heads > 65535)
    return SLS_ERR_UNSUPPORTED;
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(c, s, code, p, table, pool, stream)
                           : launch<__half>(c, s, code, p, table, pool, stream);
}

}  // namespace sls
