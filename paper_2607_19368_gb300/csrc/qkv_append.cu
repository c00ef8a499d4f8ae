// New queries and keys normalised for each head and rotated by their positions,
// keys and values appended to the paged cache, in one pass:
//   y = w x / sqrt(mean(x^2) + eps);  pair (a, b) of y turned by t = p f_i.
//
// A copy bound by HBM bandwidth with ten operations an element on the way.  A
// CTA takes a few tokens and all (or, for few tokens, a share) of their heads:
// the cosines and sines of a token are formed once in shared memory and serve
// all of its heads.  A (token, head) row is 16 lanes of one 16-byte vector each
// (8 lanes for heads of up to 64), four rows in flight per lane; the sum of
// squares stays within the row's lanes, and the partner of an element is in the
// lane half a rotation away (a shuffle), or, where the halves are no multiple of
// a vector, read again from the row.
#include <algorithm>

#include "attention.cuh"

namespace sls {

namespace {

constexpr int QA_T = 256;
constexpr int QA_TOKENS = 8;   // tokens of a CTA
constexpr int QA_ROWS = 4;     // rows in flight per lane group
constexpr int QA_MAX_PAIRS = SLS_MAX_HEAD_DIM / 2;

// cos and sin of p * f.  The product is held as a rounded float32 and its exact
// remainder (one fused multiply-add); Cody and Waite's reduction (W. J. Cody and
// W. Waite, "Software Manual for the Elementary Functions", 1980) takes multiples
// of 2 pi off it, 2 pi split into three float32 parts, each the rounding of what
// the previous ones leave: with |p f| below 2^24 the first step is exact, and the
// angle is right to a few 2^-24 at any position, where the rounded product alone
// is off by up to 2^-24 |p f|.
SLS_DEV float2 turn(float p, float f) {
  const float x = __fmul_rn(p, f);
  const float rest = __fmaf_rn(p, f, -x);
  const float k = rintf(x * 0.15915494309189535f);
  float r = __fmaf_rn(-k, 0x1.921fb6p+2f, x);
  r = __fmaf_rn(-k, -0x1.777a5cp-23f, r);
  r = __fmaf_rn(-k, -0x1.ee59dap-48f, r);
  r += rest;
  float s, c;
  sincosf(fabsf(x) < 0x1p24f ? r : x, &s, &c);
  return make_float2(c, s);
}

// L lanes per row
template <typename E, int L>
__global__ void __launch_bounds__(QA_T)
qkv_append_kernel(const __grid_constant__ AppendArgs a, int heads_per_cta) {
  __shared__ float2 s_turn[QA_TOKENS][QA_MAX_PAIRS];  // (cos, sin) * scale
  __shared__ int64_t s_slot[QA_TOKENS];               // byte offset of the token's slot, or -1
  __shared__ float s_pos[QA_TOKENS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t0 = (int64_t)blockIdx.x * QA_TOKENS;
  const int nt = (int)min((int64_t)QA_TOKENS, a.T - t0);
  const CacheView& c = a.c;

  // where each token goes: its sequence is the number of sequences that end at
  // or before it
  for (int i = warp; i < nt; i += QA_T / 32) {
    const int64_t t = t0 + i;
    int s = (int)t;
    if (a.cu) {
      int ended = 0;
      for (int b = lane; b < c.B; b += 32) ended += (a.cu[b + 1] <= t);
      s = __reduce_add_sync(0xffffffffu, ended);
    }
    if (lane == 0) {
      int64_t idx = -1, slot = -1;
      if (s < c.B) {
        const int64_t m = c.kv_lens[s];
        idx = a.cu ? m - (int64_t)a.cu[s + 1] + t : m - 1;
        if (a.cu && t < a.cu[s]) idx = -1;  // before the first sequence
        const int64_t col = idx >> c.page_shift;
        if (idx >= 0 && col < c.max_pages) {
          const int64_t page = c.table[s * c.table_ld + col];
          if (page >= 0 && page < c.num_pages)
            slot = page * c.page_b + (idx & ((1 << c.page_shift) - 1)) * c.slot_b;
        }
      }
      s_slot[i] = slot;
      s_pos[i] = a.positions ? (float)a.positions[t] : (float)idx;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nt * a.pairs; i += QA_T) {
    const int tok = i / a.pairs, pr = i - tok * a.pairs;
    const float2 cs = turn(s_pos[tok], a.inv_freq[pr]);
    s_turn[tok][pr] = make_float2(cs.x * a.rope_scale, cs.y * a.rope_scale);
  }
  __syncthreads();

  const int heads = a.q_heads + 2 * c.kv_heads;  // queries, keys, values
  const int h0 = blockIdx.y * heads_per_cta;
  const int nh = min(heads_per_cta, heads - h0);
  const int rows = nt * nh;
  const int l = threadIdx.x & (L - 1), grp = threadIdx.x / L;
  constexpr int GROUPS = QA_T / L;
  const int e0 = 8 * l;
  const bool on = e0 < c.head_dim;
  const float inv_n = 1.f / (float)c.head_dim;

  for (int r0 = grp; r0 - grp < rows; r0 += GROUPS * QA_ROWS) {
    uint4 raw[QA_ROWS];
    const char* src[QA_ROWS];
#pragma unroll
    for (int u = 0; u < QA_ROWS; ++u) {
      const int r = r0 + u * GROUPS;
      raw[u] = make_uint4(0, 0, 0, 0);
      src[u] = nullptr;
      if (r < rows) {
        const int tok = r / nh;
        const int h = h0 + r - tok * nh;
        const int64_t t = t0 + tok;
        const RowsView& v = h < a.q_heads ? a.q : (h < a.q_heads + c.kv_heads ? a.k : a.v);
        const int hh = h < a.q_heads
                           ? h
                           : (h < a.q_heads + c.kv_heads ? h - a.q_heads
                                                         : h - a.q_heads - c.kv_heads);
        src[u] = v.data + t * v.token_b + hh * v.head_b;
        if (on) raw[u] = *reinterpret_cast<const uint4*>(src[u] + 2 * e0);
      }
    }
#pragma unroll
    for (int u = 0; u < QA_ROWS; ++u) {
      const int r = r0 + u * GROUPS;
      const bool live = r < rows;
      const int tok = live ? r / nh : 0;
      const int h = live ? h0 + r - tok * nh : 0;
      const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + c.kv_heads;
      uint4 res = raw[u];
      float x[8], y[8];
      widen8<E>(raw[u], x);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __fmaf_rn(x[e], x[e], ss);
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const E* w = reinterpret_cast<const E*>(is_q ? a.q_weight : a.k_weight);
      const float f = w ? rsqrtf(__fmaf_rn(ss, inv_n, a.eps)) : 1.f;
      // the partner elements, raw: half a rotation away
      const bool first = e0 < a.pairs;
      const bool whole = (a.pairs & 7) == 0;
      uint4 other = raw[u];
      if (!a.interleaved && a.pairs > 0 && whole) {
        const int from = (lane & ~(L - 1)) + ((first ? l + (a.pairs >> 3) : l - (a.pairs >> 3)) &
                                              (L - 1));
        other.x = __shfl_sync(0xffffffffu, raw[u].x, from);
        other.y = __shfl_sync(0xffffffffu, raw[u].y, from);
        other.z = __shfl_sync(0xffffffffu, raw[u].z, from);
        other.w = __shfl_sync(0xffffffffu, raw[u].w, from);
      }
      if (live && on && !is_v) {
        if (w) {
          float g[8];
          widen8<E>(*reinterpret_cast<const uint4*>(w + e0), g);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= f * g[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e];
        if (e0 < 2 * a.pairs) {
          if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const int pr = (e0 + e) >> 1;
              if (pr < a.pairs) {
                const float2 cs = s_turn[tok][pr];
                y[e] = x[e] * cs.x - x[e + 1] * cs.y;
                y[e + 1] = x[e + 1] * cs.x + x[e] * cs.y;
              }
            }
          } else if (whole) {
            float p[8];
            widen8<E>(other, p);
            const int pe = first ? e0 + a.pairs : e0 - a.pairs;
            if (w) {
              float g[8];
              widen8<E>(*reinterpret_cast<const uint4*>(w + pe), g);
#pragma unroll
              for (int e = 0; e < 8; ++e) p[e] *= f * g[e];
            }
            const int pr = first ? e0 : pe;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 cs = s_turn[tok][pr + e];
              y[e] = first ? x[e] * cs.x - p[e] * cs.y : x[e] * cs.x + p[e] * cs.y;
            }
          } else {
            for (int e = 0; e < 8; ++e) {
              const int i = e0 + e;
              if (i >= 2 * a.pairs) break;
              const int j = i < a.pairs ? i + a.pairs : i - a.pairs;
              float p = (float)reinterpret_cast<const E*>(src[u])[j];
              if (w) p *= f * (float)w[j];
              const float2 cs = s_turn[tok][min(i, j)];
              y[e] = i < a.pairs ? x[e] * cs.x - p * cs.y : x[e] * cs.x + p * cs.y;
            }
          }
        }
        res = narrow8<E>(y);
      }
      __syncwarp();  // partners are read before a row is written in place
      if (live && on) {
        if (is_q) {
          *reinterpret_cast<uint4*>(a.out.data + (t0 + tok) * a.out.token_b + h * a.out.head_b +
                                    2 * e0) = res;
        } else if (s_slot[tok] >= 0) {
          const int hh = h - a.q_heads - (is_v ? c.kv_heads : 0);
          *reinterpret_cast<uint4*>((is_v ? c.v : c.k) + s_slot[tok] + hh * c.head_b + 2 * e0) =
              res;
        }
      }
    }
  }
}

}  // namespace

int launch_qkv_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
  if (a.T == 0) return SLS_OK;
  const int heads = a.q_heads + 2 * a.c.kv_heads;
  const int64_t tiles = (a.T + QA_TOKENS - 1) / QA_TOKENS;
  if (tiles > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  // few tokens: their heads are spread over more CTAs
  const int share = tiles >= 256 ? 1 : (int)std::min<int64_t>((256 + tiles - 1) / tiles, heads);
  const int per = (heads + share - 1) / share;
  const dim3 grid((unsigned)tiles, (unsigned)((heads + per - 1) / per));
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == SLS_BF16) {
    if (narrow) qkv_append_kernel<__nv_bfloat16, 8><<<grid, QA_T, 0, stream>>>(a, per);
    else qkv_append_kernel<__nv_bfloat16, 16><<<grid, QA_T, 0, stream>>>(a, per);
  } else {
    if (narrow) qkv_append_kernel<__half, 8><<<grid, QA_T, 0, stream>>>(a, per);
    else qkv_append_kernel<__half, 16><<<grid, QA_T, 0, stream>>>(a, per);
  }
  SLS_LAUNCH_CHECK();
  return SLS_OK;
}

}  // namespace sls
