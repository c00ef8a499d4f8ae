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
constexpr int Q8_FEW = 2;  // new tokens of a block up to which a job is one group's

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

// A lane's sixteen elements of a row of keys or values: normalised and rotated.
template <typename E, int L>
struct Q8Lane {
  const AppendArgs& a;
  const float2* s_turn;  // (slot, element of a lane's pairs, lane): cos and sin times the scale
  int l;
  bool on;
  unsigned mates;
  uint4 w[2], wp[2];     // weights of this lane's elements and of their partners

  // Pairs lie so that the lanes of a row read neighbours: a lane's pairs are sixteen in a row, or
  // eight where a pair is two elements side by side; a few float2 more a slot part the rows.
  SLS_DEV static int width(const AppendArgs& a) { return a.interleaved ? 8 : 16; }
  SLS_DEV static int lanes(const AppendArgs& a) {
    return a.interleaved ? (a.pairs + 7) >> 3 : (a.pairs + 15) >> 4;
  }

  SLS_DEV Q8Lane(const AppendArgs& args, const float2* turns, int lane, int l_)
      : a(args), s_turn(turns), l(l_), on(16 * l_ < args.c.head_dim),
        mates(((1u << L) - 1) << (lane & ~(L - 1))) {
    const E* kw = reinterpret_cast<const E*>(a.k_weight);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      w[v] = wp[v] = make_uint4(0, 0, 0, 0);
      if (!kw || !on) continue;
      const int i0 = 16 * l + 8 * v;
      w[v] = *reinterpret_cast<const uint4*>(kw + i0);
      if (!a.interleaved && i0 < 2 * a.pairs) partner(kw, i0, wp[v]);
    }
  }

  // elements i0 .. i0 + 7 of the other half of the rotated part (zeros past it)
  SLS_DEV void partner(const E* row, int i0, uint4& u) const {
    const int pairs = a.pairs;
    if ((pairs & 7) == 0) {
      u = *reinterpret_cast<const uint4*>(row + (i0 < pairs ? i0 + pairs : i0 - pairs));
      return;
    }
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e;
      x[e] = i < 2 * pairs ? reinterpret_cast<const uint16_t*>(row)[i < pairs ? i + pairs : i - pairs]
                           : 0u;
    }
    u = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
  }

  SLS_DEV void load(const char* p, uint4 (&u)[2]) const {
    u[0] = u[1] = make_uint4(0, 0, 0, 0);
    if (!on) return;
    u[0] = *reinterpret_cast<const uint4*>(p + 32 * l);
    u[1] = *reinterpret_cast<const uint4*>(p + 32 * l + 16);
  }

  // u: the row at p, loaded; y: its elements; returns the largest finite size
  SLS_DEV float row(const uint4 (&u)[2], const char* p, bool keys, int slot, float (&y)[16]) const {
    const E* xs = reinterpret_cast<const E*>(p);
    const int pairs = a.pairs;
    uint4 up[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    const bool turned = keys && 16 * l < 2 * pairs;
    if (turned && !a.interleaved) {
#pragma unroll
      for (int v = 0; v < 2; ++v)
        if (16 * l + 8 * v < 2 * pairs) partner(xs, 16 * l + 8 * v, up[v]);
    }
    float z[8];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      widen8<E>(u[v], z);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[8 * v + e] = z[e];
    }
    float norm = 1.f;
    const bool weighed = keys && a.k_weight != nullptr;
    if (weighed) {
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) s0 = __fmaf_rn(y[e], y[e], s0), s1 = __fmaf_rn(y[e + 1], y[e + 1], s1);
      s0 += s1;
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) s0 += __shfl_xor_sync(mates, s0, o);
      norm = rsqrtf(__fmaf_rn(s0, 1.f / (float)a.c.head_dim, a.eps));
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        widen8<E>(w[v], z);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[8 * v + e] *= norm * z[e];
      }
    }
    if (turned) {
      const int nl = lanes(a), stride = width(a) * nl + 4;
      const float2* tt = s_turn + slot * stride;
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          if (8 * l + e / 2 >= pairs) continue;
          const float2 cs = tt[(e / 2) * nl + l];
          const float x0 = y[e], x1 = y[e + 1];
          y[e] = x0 * cs.x - x1 * cs.y;
          y[e + 1] = x1 * cs.x + x0 * cs.y;
        }
      } else {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int i0 = 16 * l + 8 * v;
          if (i0 >= 2 * pairs) continue;
          float zw[8];
          widen8<E>(up[v], z);
          widen8<E>(wp[v], zw);
          if ((pairs & 7) == 0) {
            const bool low = i0 < pairs;
            const int p0 = low ? i0 : i0 - pairs;
            const float2* t8 = tt + (p0 & 15) * nl + (p0 >> 4);
            const float sign = low ? -1.f : 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 cs = t8[e * nl];
              const float x = weighed ? z[e] * (norm * zw[e]) : z[e];
              y[8 * v + e] = y[8 * v + e] * cs.x + sign * (x * cs.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int i = i0 + e;
              if (i >= 2 * pairs) continue;
              const bool low = i < pairs;
              const int pr = low ? i : i - pairs;
              const float2 cs = tt[(pr & 15) * nl + (pr >> 4)];
              const float x = weighed ? z[e] * (norm * zw[e]) : z[e];
              y[8 * v + e] = y[8 * v + e] * cs.x + (low ? -x : x) * cs.y;
            }
          }
        }
      }
    }
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = fabsf(y[e]);
      if (x <= 3.402823466e38f) most = fmaxf(most, x);
    }
    return most;
  }
};

// E: input type; C: codes; L: lanes of a row (16 elements each); K: rows a lane holds
template <typename E, typename C, int L, int K>
__global__ void __launch_bounds__(Q8_T, K <= 2 ? 2 : 1)
kv_append_q8_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ ScaleView sv,
                    int tile, int jobs_per_cta) {
  extern __shared__ float2 s_turn[];
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

  at_go();
  at_wait_ahead();
  const Q8Lane<E, L> me(a, s_turn, lane, l);
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
    while (row < min(at.end, t_end)) {
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
      if (j_first < c.kv_heads && a.pairs > 0) {
        const int wd = me.width(a), nl = me.lanes(a), stride = wd * nl + 4;
        for (int i = threadIdx.x; i < (hi - lo) * a.pairs; i += Q8_T) {
          const int k = i / a.pairs, pr = i - k * a.pairs;
          const int p = a.positions ? a.positions[row0 + lo + k] : (int)(start + lo + k);
          const float2 cs = turn(p, a.inv_freq[pr]);
          s_turn[(lo + k) * stride + (pr & (wd - 1)) * nl + pr / wd] =
              make_float2(cs.x * a.rope_scale, cs.y * a.rope_scale);
        }
      }
      __syncthreads();
      auto source = [&](int j, int slot) {
        const bool keys = j < c.kv_heads;
        const RowsView& src = keys ? a.k : a.v;
        return src.data + (row0 + slot) * src.token_b + (keys ? j : j - c.kv_heads) * src.head_b;
      };
      auto scale_at = [&](int j) {
        return j < c.kv_heads ? sv.k + sc + j * sv.head : sv.v + sc + (j - c.kv_heads) * sv.head;
      };
      auto codes_at = [&](int j) {
        return (j < c.kv_heads ? c.k + j * c.head_b : c.v + (j - c.kv_heads) * c.head_b) +
               page * c.page_b + slot0 * c.slot_b + 16 * l;
      };
      auto again = [&](char* d, float by) {
        float z[16];
        codes_float<C>(*reinterpret_cast<const uint4*>(d), z);
        *reinterpret_cast<uint4*>(d) = to_codes16<C>(z, by);
      };
      if (hi - lo <= Q8_FEW) {
        // ---- few new tokens: a job is one group's, all jobs at once
        for (int j = j_first + grp; j < j_end; j += NG) {
          const bool keys = j < c.kv_heads;
          float y[16], most = 0.f;
          uint4 u[2];
          for (int slot = lo; slot < hi; ++slot) {
            me.load(source(j, slot), u);
            most = fmaxf(most, me.row(u, source(j, slot), keys, slot, y));
          }
#pragma unroll
          for (int o = L / 2; o > 0; o >>= 1)
            most = fmaxf(most, __shfl_xor_sync(me.mates, most, o));
          float* sp = scale_at(j);
          const float was = lo > 0 ? *sp : 0.f;
          const float now = fmaxf(code_scale<C>(most), was), by = 1.f / now;
          char* d = codes_at(j);
          for (int slot = lo; slot < hi; ++slot) {
            if (hi - lo > 1) {
              me.load(source(j, slot), u);
              me.row(u, source(j, slot), keys, slot, y);
            }
            if (me.on) *reinterpret_cast<uint4*>(d + slot * c.slot_b) = to_codes16<C>(y, by);
          }
          if (me.on && now > was)
            for (int slot = 0; slot < lo; ++slot) again(d + slot * c.slot_b, was * by);
          __syncwarp(me.mates);  // every lane has read the old scale
          if (l == 0 && now != was) *sp = now;
        }
        continue;
      }
      // the next job's rows are on their way while one is worked on
      uint4 u[K][2];
      auto fetch = [&](int j) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int slot = grp % per_job + k * per_job;
          if (j < j_end && slot >= lo && slot < hi) me.load(source(j, slot), u[k]);
        }
      };
      fetch(j_first + grp / per_job);
      for (int j0 = j_first; j0 < j_end; j0 += together) {
        const int j = j0 + grp / per_job;
        const bool live = j < j_end, keys = j < c.kv_heads;
        float y[K][16];
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int slot = grp % per_job + k * per_job;
          // whole groups of L lanes take the branch or leave it
          if (live && slot >= lo && slot < hi)
            most = fmaxf(most, me.row(u[k], source(j, slot), keys, slot, y[k]));
        }
        fetch(j + together);
        // the rows of a warp are one head's: a block has at least as many slots as a warp rows.
        // The old scale is read in front of the barrier, behind which it is written.
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
        const float was = live && lo > 0 ? *scale_at(j) : 0.f;
        if (lane == 0) s_most[parity][warp] = most;
        __syncthreads();
        const int wj = per_job * L / 32, w0 = warp / wj * wj;
        for (int i = 0; i < wj; ++i) most = fmaxf(most, s_most[parity][w0 + i]);
        parity ^= 1;
        if (!live) continue;
        const float now = fmaxf(code_scale<C>(most), was), by = 1.f / now;
        char* d = codes_at(j);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int slot = grp % per_job + k * per_job;
          if (!me.on || slot >= hi) continue;
          if (slot >= lo) *reinterpret_cast<uint4*>(d + slot * c.slot_b) = to_codes16<C>(y[k], by);
          else if (now > was) again(d + slot * c.slot_b, was * by);
        }
        if (grp % per_job == 0 && l == 0 && now != was) *scale_at(j) = now;
      }
    }
  }
}

template <typename E, typename C, int L>
int launch(const AppendArgs& a, const ScaleView& s, cudaStream_t stream) {
  const int blk = 1 << s.shift, jobs = 2 * a.c.kv_heads;
  // a block's tokens for a CTA, or as many as a sequence has new ones on average, and heads
  // shared out until there are some 1200 CTAs (eight for each of 152 SMs)
  int tile = blk;
  while (tile > 1 && a.T < (int64_t)tile * a.c.B) tile /= 2;
  const int64_t tiles = (a.T + tile - 1) / tile;
  // jobs that a CTA has in flight
  const int together = tile <= Q8_FEW ? Q8_T / L : std::max(1, Q8_T / L / blk);
  const int passes = (jobs + together - 1) / together;
  const int share = (int)std::max<int64_t>(1, std::min<int64_t>((1216 + tiles - 1) / tiles, passes));
  const int per = (passes + share - 1) / share * together;
  const dim3 grid((unsigned)tiles, (unsigned)((jobs + per - 1) / per));
  const int width = a.interleaved ? 8 : 16;
  const size_t smem = a.pairs == 0 ? 0
                      : (size_t)blk * ((a.pairs + width - 1) / width * width + 4) * sizeof(float2);
  const int rows = blk * L / Q8_T;
  auto kern = rows <= 1 ? kv_append_q8_kernel<E, C, L, 1>
              : rows == 2 ? kv_append_q8_kernel<E, C, L, 2> : kv_append_q8_kernel<E, C, L, L / 2>;
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
