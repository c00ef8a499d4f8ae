// Attention over the paged cache, one warp per (token, query head) row:
//   o = sum_j exp(s_j - max) v_j / sum_j exp(s_j - max),  s_j = scale q . k_j,
// with the running maximum and sum of a softmax taken key by key.  Every lane
// holds four elements of the head.
#include <algorithm>

#include "attention.cuh"

namespace sls {

namespace {

constexpr int AS_T = 256;

template <typename E>
__global__ void __launch_bounds__(AS_T)
attention_simt_kernel(const __grid_constant__ AttnArgs a) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  const int64_t rows = a.T * a.q_heads;
  const int64_t step = (int64_t)gridDim.x * (AS_T / 32);
  const int group = a.q_heads / c.kv_heads;
  const int e0 = 4 * lane;
  const bool on = e0 < c.head_dim;
  for (int64_t r = (int64_t)blockIdx.x * (AS_T / 32) + (threadIdx.x >> 5); r < rows; r += step) {
    const int64_t t = r / a.q_heads;
    const int h = (int)(r - t * a.q_heads);
    int s = (int)t;
    int64_t keys;
    if (a.cu) {
      int ended = 0;
      for (int b = lane; b < c.B; b += 32) ended += (a.cu[b + 1] <= t);
      s = __reduce_add_sync(0xffffffffu, ended);
      if (s >= c.B || t < a.cu[s]) continue;
    }
    keys = cache_len(c, s);
    if (a.cu && a.causal) keys = min(keys, (int64_t)c.kv_lens[s] - a.cu[s + 1] + t + 1);
    float q[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f};
    if (on) {
      const uint2 u =
          *reinterpret_cast<const uint2*>(a.q.data + t * a.q.token_b + h * a.q.head_b + 2 * e0);
      const float2 f0 = Half2<E>::widen(u.x), f1 = Half2<E>::widen(u.y);
      q[0] = f0.x * a.scale, q[1] = f0.y * a.scale, q[2] = f1.x * a.scale, q[3] = f1.y * a.scale;
    }
    float mx = -INFINITY, l = 0.f;
    for (int64_t j = 0; j < keys; ++j) {
      const int64_t page = c.table[s * c.table_ld + (j >> c.page_shift)];
      float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
      if (on && page >= 0 && page < c.num_pages) {
        const int64_t off = page * c.page_b + (j & ((1 << c.page_shift) - 1)) * c.slot_b +
                            (h / group) * c.head_b + 2 * e0;
        const uint2 ku = *reinterpret_cast<const uint2*>(c.k + off);
        const uint2 vu = *reinterpret_cast<const uint2*>(c.v + off);
        const float2 k0 = Half2<E>::widen(ku.x), k1 = Half2<E>::widen(ku.y);
        const float2 v0 = Half2<E>::widen(vu.x), v1 = Half2<E>::widen(vu.y);
        k[0] = k0.x, k[1] = k0.y, k[2] = k1.x, k[3] = k1.y;
        v[0] = v0.x, v[1] = v0.y, v[2] = v1.x, v[3] = v1.y;
      }
      float d = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
      const float mn = fmaxf(mx, d);
      const float base = mn == -INFINITY ? 0.f : mn;
      const float corr = __expf(mx - base), p = __expf(d - base);
      l = l * corr + p;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] * corr + p * v[e];
      mx = mn;
    }
    const float inv = keys > 0 ? 1.f / l : 0.f;
    if (on)
      *reinterpret_cast<uint2*>(a.out.data + t * a.out.token_b + h * a.out.head_b + 2 * e0) =
          make_uint2(Half2<E>::narrow(o[0] * inv, o[1] * inv),
                     Half2<E>::narrow(o[2] * inv, o[3] * inv));
  }
}

}  // namespace

int launch_attention(const AttnArgs& a, int dtype, cudaStream_t stream) {
  const int64_t rows = a.T * a.q_heads;
  if (rows == 0) return SLS_OK;
  const int grid = (int)std::min<int64_t>((rows + 7) / 8, 152 * 8);
  if (dtype == SLS_BF16) attention_simt_kernel<__nv_bfloat16><<<grid, AS_T, 0, stream>>>(a);
  else attention_simt_kernel<__half><<<grid, AS_T, 0, stream>>>(a);
  SLS_LAUNCH_CHECK();
  return SLS_OK;
}

}  // namespace sls
