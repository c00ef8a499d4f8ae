// New keys (normalised, rotated) and values as 8-bit codes: a power-of-two scale for each block
// of a page's slots and key head,
//   s' = max(s, 2^e), 2^e the least with max|y| <= Q 2^e,   c = round(y / s'),
// s the scale of a block that holds earlier tokens, whose codes c become round(c s / s') when
// it grows.
//
// A CTA takes blocks whose first new token lies among its `tile` packed tokens, one after the
// other, and all or a share of their heads: cosines and sines are formed once for all heads.
// A lane holds sixteen elements of a token's head (its code is one 16-byte store), four or
// eight lanes a row; rows stay in registers between the maximum over the block and the codes,
// so that inputs are read once.  Warps of one head exchange maxima through shared memory.
//
// The queries go through the 16-bit append's kernel, with no key heads.
#include <algorithm>

#include "attention_turn.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int Q8_T = 256;

// Where a packed token goes.
struct Q8Place {
  int seq;
  int64_t begin, end;  // the sequence's placed new tokens: packed rows [begin, end)
  int64_t index0;      // cache index of row `begin`
};

SLS_DEV Q8Place q8_place(const AppendArgs& a, int s) {
  const CacheView& c = a.c;
  const int64_t m = c.kv_lens[s];
  int64_t b = s, e = s + 1;
  if (a.cu) seq_rows(a.cu, s, a.T, b, e);
  // the same cut as for the rows: tokens before index 0 or past the table have no place.  The
  // last row of a sequence that the packing cuts short keeps its index.
  const int64_t last = a.cu ? (int64_t)a.cu[s + 1] : e;
  const int64_t room = (int64_t)c.max_pages << c.page_shift;
  int64_t x = m - last + b;  // index of row b
  if (x < 0) b -= x, x = 0;
  e = min(e, b + max((int64_t)0, room - x));
  return Q8Place{s, b, max(b, e), x};
}

// E: input type; C: codes; L: lanes of a row (16 elements each); K: rows a lane holds
template <typename E, typename C, int L, int K>
__global__ void __launch_bounds__(Q8_T)
kv_append_q8_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ ScaleView sv,
                    int tile, int jobs_per_cta) {
  extern __shared__ float2 s_turn[];     // block tokens x pairs: (cos, sin) * scale
  __shared__ float s_most[2][Q8_T / 32];
  __shared__ int s_ended[Q8_T / 32];
  constexpr int NG = Q8_T / L;           // rows in flight
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = threadIdx.x / L, l = threadIdx.x % L;
  const int blk = 1 << sv.shift;
  const int per_job = min(blk, NG);      // groups of a job (one head of keys or of values)
  const int together = NG / per_job;     // jobs in flight
  const int jobs = 2 * c.kv_heads;
  const int j_first = blockIdx.y * jobs_per_cta, j_end = min(jobs, j_first + jobs_per_cta);
  const int64_t t_end = min(a.T, ((int64_t)blockIdx.x + 1) * tile);
  int64_t t = (int64_t)blockIdx.x * tile;
  const bool on = 16 * l < c.head_dim;
  const int pairs = a.pairs;

  at_go();
  at_wait_ahead();
  int seq = (int)t;
  if (a.cu) {
    int ended = 0;
    for (int b = threadIdx.x; b < c.B; b += Q8_T) ended += a.cu[b + 1] <= t;
    ended = __reduce_add_sync(0xffffffffu, ended);
    if (lane == 0) s_ended[warp] = ended;
    __syncthreads();
    seq = 0;
    for (int w = 0; w < Q8_T / 32; ++w) seq += s_ended[w];
  }
  int parity = 0;
  for (; seq < c.B; ++seq) {
    const Q8Place at = q8_place(a, seq);
    if (a.cu ? (int64_t)a.cu[seq] >= t_end : seq >= t_end) break;
    // blocks whose first new token is a row of [t, t_end)
    int64_t row = max(at.begin, t);
    int64_t idx = at.index0 + row - at.begin;
    if (row > at.begin && (idx & (blk - 1))) {
      row += blk - (idx & (blk - 1));
      idx = at.index0 + row - at.begin;
    }
    for (; row < min(at.end, t_end);) {
      const int64_t start = idx & ~(int64_t)(blk - 1);
      const int lo = (int)(idx - start);                             // first new slot
      const int hi = (int)min((int64_t)blk, lo + at.end - row);      // past the last
      const int64_t row0 = row - lo;                                 // row of the block's slot 0
      row += hi - lo;
      idx += hi - lo;
      const int64_t page = c.table[seq * c.table_ld + (start >> c.page_shift)];
      if (page < 0 || page >= c.num_pages) continue;
      const int slot0 = (int)(start & ((1 << c.page_shift) - 1));
      const int64_t sc = page * sv.page + (slot0 >> sv.shift) * sv.block;
      // the turns of the block's new tokens, for all heads of keys
      __syncthreads();
      if (j_first < c.kv_heads)
        for (int i = threadIdx.x; i < (hi - lo) * pairs; i += Q8_T) {
          const int k = i / pairs, pr = i - k * pairs;
          const int p = a.positions ? a.positions[row0 + lo + k] : (int)(start + lo + k);
          const float2 cs = turn(p, a.inv_freq[pr]);
          s_turn[(lo + k) * pairs + pr] = make_float2(cs.x * a.rope_scale, cs.y * a.rope_scale);
        }
      __syncthreads();
      for (int j0 = j_first; j0 < j_end; j0 += together) {
        const int j = j0 + grp / per_job;
        const bool live = j < j_end;
        const bool keys = j < c.kv_heads;
        const int h = keys ? j : j - c.kv_heads;
        const RowsView& src = keys ? a.k : a.v;
        const E* w = keys ? reinterpret_cast<const E*>(a.k_weight) : nullptr;
        float y[K][16];
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int slot = grp % per_job + k * per_job;
#pragma unroll
          for (int e = 0; e < 16; ++e) y[k][e] = 0.f;
          // whole groups of L lanes take the branch or leave it
          if (live && slot >= lo && slot < hi) {
            const char* p = src.data + (row0 + slot) * src.token_b + h * src.head_b;
            const E* xs = reinterpret_cast<const E*>(p);
            if (on) {
              float z[8];
              widen8<E>(*reinterpret_cast<const uint4*>(p + 32 * l), z);
#pragma unroll
              for (int e = 0; e < 8; ++e) y[k][e] = z[e];
              widen8<E>(*reinterpret_cast<const uint4*>(p + 32 * l + 16), z);
#pragma unroll
              for (int e = 0; e < 8; ++e) y[k][8 + e] = z[e];
            }
            float norm = 1.f;
            if (w) {
              float ss = 0.f;
#pragma unroll
              for (int e = 0; e < 16; ++e) ss = __fmaf_rn(y[k][e], y[k][e], ss);
              const unsigned mates = ((L == 32 ? 0u : 1u << L) - 1) << (lane & ~(L - 1));
#pragma unroll
              for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mates, ss, o);
              norm = rsqrtf(__fmaf_rn(ss, 1.f / (float)c.head_dim, a.eps));
#pragma unroll
              for (int e = 0; e < 16; ++e) y[k][e] *= norm * (on ? (float)w[16 * l + e] : 0.f);
            }
            if (keys && on && 16 * l < 2 * pairs) {
              const float2* tt = s_turn + slot * pairs;
              if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                  const int pr = 8 * l + e / 2;
                  if (pr >= pairs) continue;
                  const float2 cs = tt[pr];
                  const float u = y[k][e], v = y[k][e + 1];
                  y[k][e] = u * cs.x - v * cs.y;
                  y[k][e + 1] = v * cs.x + u * cs.y;
                }
              } else {
                // partners are read from the row again, by vectors where pairs are whole ones
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                  const int i0 = 16 * l + 8 * v;
                  if (i0 >= 2 * pairs) continue;
                  float z[8], wz[8];
                  if ((pairs & 7) == 0) {
                    const int o0 = i0 < pairs ? i0 + pairs : i0 - pairs;
                    widen8<E>(*reinterpret_cast<const uint4*>(xs + o0), z);
                    if (w) widen8<E>(*reinterpret_cast<const uint4*>(w + o0), wz);
                  } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                      const int i = i0 + e, o = i < pairs ? i + pairs : i - pairs;
                      const bool in = i < 2 * pairs;
                      z[e] = in ? (float)xs[o] : 0.f;
                      wz[e] = in && w ? (float)w[o] : 0.f;
                    }
                  }
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const int i = i0 + e;
                    if (i >= 2 * pairs) continue;
                    const bool low = i < pairs;
                    const float2 cs = tt[low ? i : i - pairs];
                    const float x = y[k][8 * v + e], u = w ? z[e] * (norm * wz[e]) : z[e];
                    y[k][8 * v + e] = low ? x * cs.x - u * cs.y : x * cs.x + u * cs.y;
                  }
                }
              }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float z = fabsf(y[k][e]);
              if (z <= 3.402823466e38f) most = fmaxf(most, z);
            }
          }
        }
        // the rows of a warp are one head's: a block has at least as many slots as a warp rows.
        // The old scale is read in front of the barrier, behind which it is written.
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
        float* sp = (keys ? sv.k : sv.v) + sc + h * sv.head;
        const float was = live && lo > 0 ? *sp : 0.f;
        if (lane == 0) s_most[parity][warp] = most;
        __syncthreads();
        const int wj = per_job * L / 32, w0 = warp / wj * wj;
        for (int i = 0; i < wj; ++i) most = fmaxf(most, s_most[parity][w0 + i]);
        parity ^= 1;
        if (!live) continue;
        const float now = fmaxf(code_scale<C>(most), was);
        const float by = 1.f / now;
        char* dst = (keys ? c.k : c.v) + page * c.page_b + slot0 * c.slot_b + h * c.head_b;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int slot = grp % per_job + k * per_job;
          if (!on || slot >= hi) continue;
          uint4* d = reinterpret_cast<uint4*>(dst + slot * c.slot_b + 16 * l);
          if (slot >= lo) {
            *d = to_codes16<C>(y[k], by);
          } else if (now > was) {
            float z[16];
            codes_float<C>(*d, z);
            *d = to_codes16<C>(z, was * by);
          }
        }
        if (grp % per_job == 0 && l == 0 && now != was) *sp = now;
      }
    }
  }
}

template <typename E, typename C, int L>
int launch(const AppendArgs& a, const ScaleView& s, cudaStream_t stream) {
  const int blk = 1 << s.shift, jobs = 2 * a.c.kv_heads;
  // as many tokens as a block has where that gives the GPU enough CTAs, down to one (single
  // tokens of many sequences), and heads shared out until there are some 600
  int tile = blk;
  while (tile > 1 && (a.T + tile - 1) / tile < 608) tile /= 2;
  const int64_t tiles = (a.T + tile - 1) / tile;
  const int together = std::max(1, Q8_T / L / blk);
  const int share = (int)std::max<int64_t>(1, std::min<int64_t>(608 / tiles, (jobs + together - 1) / together));
  int per = (jobs + share - 1) / share;
  per = (per + together - 1) / together * together;
  const dim3 grid((unsigned)tiles, (unsigned)((jobs + per - 1) / per));
  const size_t smem = (size_t)blk * a.pairs * sizeof(float2);
  const int rows = blk * L / Q8_T;
  auto kern = rows <= 1 ? kv_append_q8_kernel<E, C, L, 1>
              : rows == 2 ? kv_append_q8_kernel<E, C, L, 2> : kv_append_q8_kernel<E, C, L, 4>;
  if (smem > 48 * 1024)
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)smem));
  return at_launch(kern, grid, Q8_T, smem, 1, stream, a, s, tile, per);
}

template <typename E>
int launch(const AppendArgs& a, const ScaleView& s, int code, cudaStream_t stream) {
  if (code == SLS_I8)
    return a.c.head_dim > 64 ? launch<E, I8, 8>(a, s, stream) : launch<E, I8, 4>(a, s, stream);
  return a.c.head_dim > 64 ? launch<E, E4M3, 8>(a, s, stream) : launch<E, E4M3, 4>(a, s, stream);
}

}  // namespace

int launch_kv_append_q8(const AppendArgs& a, const ScaleView& s, int code, int dtype,
                        cudaStream_t stream) {
  if (a.T == 0) return SLS_OK;
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, s, code, stream)
                           : launch<__half>(a, s, code, stream);
}

}  // namespace sls
