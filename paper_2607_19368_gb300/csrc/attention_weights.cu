// The weight that queries place on every cached token, summed over rows i (tokens) and the
// query heads of a key head and added to a running sum:
//   w_j += sum_i exp(s_ij - m_i) / l_i,   m_i = max_j s_ij,  l_i = sum_j exp(s_ij - m_i).
//
// A column can be summed only when the rows' m and l are known, so there are two passes over
// the scores.  A CTA owns 256 cached tokens of a (sequence, key head), 32 a warp, whose keys
// stay in registers as mma.sync operands (codes become float16 once) while rows pass by,
// sixteen at a time from shared memory.  The first pass leaves a row's maximum and sum over the
// 256 tokens; a small launch joins them; the second pass forms the scores again and sums columns
// in registers, so that no sum is made by atomics: the same call gives the same bits.
//
// Where rows are few (a token for each sequence) the kernels of attention_weights_few.cu read keys
// once instead.
#include <algorithm>

#include "attention_decode.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int AW_WARPS = 8;
constexpr int AW_T = 32 * AW_WARPS;
constexpr int AW_KEYS = 32 * AW_WARPS;  // tokens of a CTA's unit
constexpr int AW_TILES = 16;            // row tiles in shared memory at a time
constexpr int AW_BLOCK = 16 * AW_TILES;

struct AwPlan {
  float2* part;   // (token, query head, unit of the sequence): maximum and sum of its tokens
  float2* stat;   // (token, query head): maximum, one over the sum
  int units;      // of the longest sequence that the table holds
};

template <typename E, typename KT>
using AwMma = typename std::conditional<std::is_same<E, KT>::value, E, __half>::type;

// first of the four elements of slice k that a lane's quarter cq of a row holds
template <bool CODES>
SLS_DEV int aw_element(int k, int cq) {
  return CODES ? 64 * (k >> 2) + 16 * cq + 4 * (k & 3) : 32 * (k >> 1) + 8 * cq + 4 * (k & 1);
}

// The packed rows of a sequence.
SLS_DEV void aw_rows(const AttnArgs& a, int seq, int64_t& q0, int64_t& q1) {
  if (a.cu) {
    seq_rows(a.cu, seq, a.T, q0, q1);
  } else {
    q0 = seq, q1 = seq + 1;
  }
}

// SUM: the second pass
template <typename E, typename KT, int HD, bool SUM>
__global__ void __launch_bounds__(AW_T, 2)
attention_weights_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ ScaleView sc,
                         const __grid_constant__ WeightView wv, const __grid_constant__ AwPlan p) {
  using M = AwMma<E, KT>;
  constexpr bool CODES = !std::is_same<E, KT>::value;
  constexpr int KS = HD / 16;
  extern __shared__ __align__(16) unsigned char smem[];
  uint4* s_q = reinterpret_cast<uint4*>(smem);                     // (tile, slice, lane)
  float* s_f = reinterpret_cast<float*>(s_q + AW_TILES * KS * 32);  // a row's factor
  int* s_see = reinterpret_cast<int*>(s_f + AW_BLOCK);              // tokens that a row sees
  float2* s_ml = reinterpret_cast<float2*>(s_see + AW_BLOCK);      // (warp, row), or (row) of stat
  __shared__ int64_t s_pre[AW_T + 1];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = lane >> 2, cq = lane & 3;
  const int group = a.q_heads / c.kv_heads;
  const float cs = a.scale * 1.4426950408889634f;

  at_wait_ahead();
  const auto count = [&](int s) { return ad_steps<AW_KEYS>(c, s); };
  const int R = ad_prefix<AW_T>(c, s_pre, nullptr, count);
  const int64_t total = s_pre[AW_T] * c.kv_heads;
  const int64_t u0 = total * blockIdx.x / gridDim.x, u1 = total * (blockIdx.x + 1) / gridDim.x;
  int64_t staged = -1;  // the rows in shared memory: sequence times key heads plus head
  for (int64_t u = u0; u < u1; ++u) {
    // units lie by sequence, key head and tokens
    int seq;
    int64_t before;
    ad_find<AW_T>(s_pre, R, u / c.kv_heads, count, seq, before);
    const int units = ad_steps<AW_KEYS>(c, seq);
    const int64_t in = u - before * c.kv_heads;
    const int h = (int)(in / units), unit = (int)(in - (int64_t)h * units);
    const int len = (int)cache_len(c, seq);
    int64_t q0, q1;
    aw_rows(a, seq, q0, q1);
    const int n = (int)(q1 - q0);
    const int64_t rows = (int64_t)n * group;
    if (rows == 0) continue;

    // ---- this warp's keys ----
    const int key0 = unit * AW_KEYS + warp * 32;
    uint32_t kf[4][KS][2];
    float ks[4];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb) {
      const int x = key0 + 8 * nb + r;
      int64_t page = -1;
      const int slot = x & ((1 << c.page_shift) - 1);
      if (x < len) page = c.table[seq * c.table_ld + (x >> c.page_shift)];
      const bool real = page >= 0 && page < c.num_pages;
      const char* k = c.k + (real ? page : 0) * c.page_b + slot * c.slot_b + h * c.head_b;
      ks[nb] = 1.f;
      if constexpr (CODES) {
        ks[nb] = real ? sc.k[page * sc.page + (slot >> sc.shift) * sc.block + h * sc.head] : 0.f;
#pragma unroll
        for (int i = 0; i < KS / 4; ++i) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (real && 64 * i + 16 * cq < c.head_dim)
            w = *reinterpret_cast<const uint4*>(k + 64 * i + 16 * cq);
          codes_half<KT>(w.x, kf[nb][4 * i][0], kf[nb][4 * i][1]);
          codes_half<KT>(w.y, kf[nb][4 * i + 1][0], kf[nb][4 * i + 1][1]);
          codes_half<KT>(w.z, kf[nb][4 * i + 2][0], kf[nb][4 * i + 2][1]);
          codes_half<KT>(w.w, kf[nb][4 * i + 3][0], kf[nb][4 * i + 3][1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (real && 32 * i + 8 * cq < c.head_dim)
            w = *reinterpret_cast<const uint4*>(k + 64 * i + 16 * cq);
          kf[nb][2 * i][0] = w.x, kf[nb][2 * i][1] = w.y;
          kf[nb][2 * i + 1][0] = w.z, kf[nb][2 * i + 1][1] = w.w;
        }
      }
      // the scale of the tokens of this lane's columns: eight tokens share a block
      if constexpr (CODES) ks[nb] = __shfl_sync(0xffffffffu, ks[nb], 0);
    }
    float col[4][2];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb) col[nb][0] = col[nb][1] = 0.f;

    for (int64_t b0 = 0; b0 < rows; b0 += AW_BLOCK) {
      const int here = (int)min((int64_t)AW_BLOCK, rows - b0);
      const int tiles = (here + 15) / 16;
      // ---- rows to shared memory, in the order of the products' operands ----
      const bool again = staged == (int64_t)seq * c.kv_heads + h && rows <= AW_BLOCK;
      if (!again) {
        __syncthreads();
        for (int tile = warp; tile < tiles; tile += AW_WARPS) {
          uint4 f[KS];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int64_t row = b0 + 16 * tile + r + 8 * x;
            const int64_t tok = row / group;
            const int g = (int)(row - tok * group);
            const char* qp = a.q.data + (q0 + tok) * a.q.token_b + (h * group + g) * a.q.head_b;
            uint2 raw[KS];
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              const int e = aw_element<CODES>(k, cq);
              raw[k] = row < rows && e < c.head_dim ? *reinterpret_cast<const uint2*>(qp + 2 * e)
                                                    : make_uint2(0u, 0u);
              const float2 y = Half2<E>::widen(raw[k].x), z = Half2<E>::widen(raw[k].y);
              top = fmaxf(fmaxf(fmaxf(top, fabsf(y.x)), fmaxf(fabsf(y.y), fabsf(z.x))), fabsf(z.y));
            }
            if constexpr (!std::is_same<E, M>::value) {
              // bfloat16 to float16: the largest element of a row to [2^14, 2^15)
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
              const int e = max(__float_as_int(top) >> 23, 16);
              const float by = __int_as_float((127 + 14 + 127 - e) << 23);
              if (cq == 0) s_f[16 * tile + r + 8 * x] = __int_as_float((e - 14) << 23);
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                const float2 y = Half2<E>::widen(raw[k].x), z = Half2<E>::widen(raw[k].y);
                raw[k].x = Half2<__half>::narrow(y.x * by, y.y * by);
                raw[k].y = Half2<__half>::narrow(z.x * by, z.y * by);
              }
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              if (x == 0) f[k].x = raw[k].x, f[k].z = raw[k].y;
              else f[k].y = raw[k].x, f[k].w = raw[k].y;
            }
          }
#pragma unroll
          for (int k = 0; k < KS; ++k) s_q[(tile * KS + k) * 32 + lane] = f[k];
        }
        for (int i = threadIdx.x; i < 16 * tiles; i += AW_T)
          s_see[i] = i >= here ? 0 : a.causal ? len - n + (int)((b0 + i) / group) + 1 : len;
        if constexpr (SUM)
          for (int i = threadIdx.x; i < here; i += AW_T) {
            const int64_t tok = (b0 + i) / group;
            s_ml[i] = p.stat[(q0 + tok) * a.q_heads + h * group + (int)(b0 + i - tok * group)];
          }
        __syncthreads();
      }
      staged = (int64_t)seq * c.kv_heads + h;

      for (int tile = 0; tile < tiles && key0 < len; ++tile) {
        float s[4][4];
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 f = s_q[(tile * KS + k) * 32 + lane];
          const uint32_t q[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
          for (int nb = 0; nb < 4; ++nb) mma16816<M>(s[nb], q, kf[nb][k][0], kf[nb][k][1]);
        }
        if constexpr (CODES) {
          const float f0 = std::is_same<E, M>::value ? 1.f : s_f[16 * tile + r];
          const float f1 = std::is_same<E, M>::value ? 1.f : s_f[16 * tile + r + 8];
#pragma unroll
          for (int nb = 0; nb < 4; ++nb) {
            s[nb][0] *= ks[nb] * f0, s[nb][1] *= ks[nb] * f0;
            s[nb][2] *= ks[nb] * f1, s[nb][3] *= ks[nb] * f1;
          }
        }
        // tokens that each of the two rows sees
        const int see0 = s_see[16 * tile + r], see1 = s_see[16 * tile + r + 8];
        bool hide[4][4] = {};
        if (!__all_sync(0xffffffffu, key0 + 32 <= min(see0, see1))) {
#pragma unroll
          for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              hide[nb][i] = key0 + 8 * nb + 2 * cq + (i & 1) >= (i < 2 ? see0 : see1);
              if (hide[nb][i]) s[nb][i] = -INFINITY;
            }
        }
        if constexpr (!SUM) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) m = fmaxf(fmaxf(m, s[nb][2 * x]), s[nb][2 * x + 1]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
              l += at_exp2((s[nb][2 * x] - base) * cs) + at_exp2((s[nb][2 * x + 1] - base) * cs);
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            if (cq == 0) s_ml[warp * AW_BLOCK + 16 * tile + r + 8 * x] = make_float2(m, l);
          }
        } else {
          const float2 m0 = s_ml[16 * tile + r], m1 = s_ml[16 * tile + r + 8];
#pragma unroll
          for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 m = i < 2 ? m0 : m1;
              const float w = at_exp2((s[nb][i] - m.x) * cs) * m.y;
              col[nb][i & 1] += hide[nb][i] ? 0.f : w;
            }
        }
      }
      if constexpr (!SUM) {
        __syncthreads();
        const int live = min(AW_WARPS, (len - unit * AW_KEYS + 31) / 32);
        for (int i = threadIdx.x; i < here; i += AW_T) {
          float m = -INFINITY, l = 0.f;
          for (int w = 0; w < live; ++w) m = fmaxf(m, s_ml[w * AW_BLOCK + i].x);
          const float base = m == -INFINITY ? 0.f : m;
          for (int w = 0; w < live; ++w) {
            const float2 x = s_ml[w * AW_BLOCK + i];
            l += x.y * at_exp2((x.x - base) * cs);
          }
          const int64_t tok = (b0 + i) / group;
          const int g = (int)(b0 + i - tok * group);
          p.part[((q0 + tok) * a.q_heads + h * group + g) * p.units + unit] = make_float2(m, l);
        }
        __syncthreads();
      }
    }
    if constexpr (SUM) {
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float w = col[nb][i];
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
          const int x = key0 + 8 * nb + 2 * cq + i;
          if (r != 0 || x >= len) continue;
          const int64_t page = c.table[seq * c.table_ld + (x >> c.page_shift)];
          if (page >= 0 && page < c.num_pages)
            wv.data[page * wv.page + h * wv.head + (x & ((1 << c.page_shift) - 1))] += w;
        }
    }
  }
}

// A warp for each row: the sequence's units in order.
__global__ void __launch_bounds__(AW_T)
attention_weights_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AwPlan p) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * AW_WARPS + (threadIdx.x >> 5);
  if (row >= a.T * a.q_heads) return;
  const int64_t t = row / a.q_heads;
  const float cs = a.scale * 1.4426950408889634f;
  at_go();
  at_wait_ahead();
  int seq = (int)t;
  if (a.cu) {
    int ended = 0;
    for (int b = lane; b < c.B; b += 32) ended += a.cu[b + 1] <= t;
    seq = __reduce_add_sync(0xffffffffu, ended);
    if (seq >= c.B || t < a.cu[seq]) return;
  }
  const int units = ad_steps<AW_KEYS>(c, seq);
  const float2* part = p.part + row * p.units;
  float m = -INFINITY, l = 0.f;
  for (int u = lane; u < units; u += 32) {
    const float2 x = part[u];
    const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.f : top;
    l = l * at_exp2((m - base) * cs) + x.y * at_exp2((x.x - base) * cs);
    m = top;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
    // the same order of the two addends in both lanes
    const float x = l * at_exp2((m - base) * cs), y = l2 * at_exp2((m2 - base) * cs);
    l = (lane & o) ? y + x : x + y;
    m = top;
  }
  if (lane == 0) p.stat[row] = make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / l);
}

int aw_units(const CacheView& c) {
  return (int)((((int64_t)c.max_pages << c.page_shift) + AW_KEYS - 1) / AW_KEYS);
}
size_t aw_part_bytes(const CacheView& c, int64_t T, int q_heads) {
  return sls_align256((size_t)T * q_heads * aw_units(c) * 8);
}

template <typename E, typename KT, int HD>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, void* workspace, cudaStream_t stream) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  AwPlan p;
  p.units = aw_units(a.c);
  p.part = (float2*)workspace;
  p.stat = (float2*)((char*)workspace + aw_part_bytes(a.c, a.T, a.q_heads));
  const int64_t most = (int64_t)a.c.B * p.units * a.c.kv_heads;
  const unsigned grid = (unsigned)std::min<int64_t>(most, 2 * sms);
  constexpr size_t rows = (size_t)AW_TILES * (HD / 16) * 512 + AW_BLOCK * 8;
  constexpr size_t smem1 = rows + AW_WARPS * AW_BLOCK * 8, smem2 = rows + AW_BLOCK * 8;
  auto first = attention_weights_kernel<E, KT, HD, false>;
  auto second = attention_weights_kernel<E, KT, HD, true>;
  SLS_CUDA_TRY(cudaFuncSetAttribute(first, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem1));
  SLS_CUDA_TRY(
      cudaFuncSetAttribute(second, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem2));
  int st = at_launch(first, dim3(grid), AW_T, smem1, 1, stream, a, s, w, p);
  if (st != SLS_OK) return st;
  const int64_t all = a.T * a.q_heads;
  st = at_launch(attention_weights_join_kernel, dim3((unsigned)((all + AW_WARPS - 1) / AW_WARPS)),
                 AW_T, 0, 1, stream, a, p);
  if (st != SLS_OK) return st;
  return at_launch(second, dim3(grid), AW_T, smem2, 1, stream, a, s, w, p);
}

template <typename E, typename KT>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, void* workspace, cudaStream_t stream) {
  return a.c.head_dim > 64 ? launch<E, KT, 128>(a, s, w, workspace, stream)
                           : launch<E, KT, 64>(a, s, w, workspace, stream);
}

template <typename E>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code, void* workspace, cudaStream_t stream) {
  return code == SLS_I8     ? launch<E, I8>(a, s, w, workspace, stream)
         : code == SLS_E4M3 ? launch<E, E4M3>(a, s, w, workspace, stream)
                            : launch<E, E>(a, s, w, workspace, stream);
}

}  // namespace

size_t attention_weights_workspace(const CacheView& c, int64_t T, int q_heads, int code) {
  if (c.B == 0 || T == 0 || c.max_pages == 0) return 0;
  if (attention_weights_few(c, T, q_heads, code))
    return attention_weights_few_workspace(c, T, q_heads);
  return aw_part_bytes(c, T, q_heads) + sls_align256((size_t)T * q_heads * 8);
}

int launch_attention_weights(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code,
                             int dtype, void* workspace, cudaStream_t stream) {
  if (a.c.B == 0 || a.T == 0 || a.c.max_pages == 0) return SLS_OK;
  if (a.T * a.q_heads > (int64_t)0x7fffffff * AW_WARPS) return SLS_ERR_UNSUPPORTED;
  if (attention_weights_few(a.c, a.T, a.q_heads, code))
    return launch_attention_weights_few(a, s, w, code, dtype, workspace, stream);
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, s, w, code, workspace, stream)
                           : launch<__half>(a, s, w, code, workspace, stream);
}

}  // namespace sls
