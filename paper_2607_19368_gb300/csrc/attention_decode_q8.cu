// One new token per sequence over a paged cache of 8-bit codes: o = softmax(scale q K^T) V with
// k = sk c^k and v = sv c^v, codes and scales read once.
//
// Bound by HBM bandwidth: 2 hd bytes a cached token and key head, against some 500 instructions
// of a warp for each 32 tokens of a head, which take half of the issue slots.  64 streams to 8192
// tokens, 32 + 8 heads of 128, int8 in pages of 16: 92.0 us, 5.5 TB/s; 3 to 131072, 40 + 8, e4m3:
// 103.2 us, 5.8 TB/s; one of 2061 tokens 7.7 us, latency.  A warp owns a (sequence, key head) at a time, its parts
// and pieces as in the 16-bit kernel, and multiplies float16 (every code is one exactly) by
// mma.sync.  What the 8 bits change:
//  * The scale of a block of tokens multiplies finished scores, and weights instead of values.  Weights
//    are then in units of their own for each head, to stay in float16's range: see q8_unit (64 streams
//    91.9 us; with one unit for all heads, the largest scale so far, 90.9, but wrong for values far apart).
//  * bfloat16 queries become float16 times a power of two for each row, which scores take back:
//    exact down to 2^-31 of the row's largest element, and to 2^-39 of it below.
//  * Keys and values are the 16-row operands, query heads the 8 columns (S^T = K Q^T, O^T = V^T
//    P^T): up to eight heads a key head take half the products, registers and exponentials that
//    they take as half of a 16-row tile, and 12 warps fit instead of 8.  Weights change sides by
//    movmatrix.
//  * An operand's registers come from whole bytes of a row: sixteen of a key, the elements of a
//    head in an order of their own (the same for queries); sixteen (or eight) of four values, bytes
//    of two keys interleaved.  No transposing load is needed.  Tokens 2 c and 2 c + 1 of an operand
//    are 2 c and (2 c ^ 4) + 1 of the cache, so that neither read meets a bank twice.
#include <algorithm>

#include "attention_decode.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr float Q8_SHIFT = 15.f;  // log2 of a factor of all weights, see the 16-bit kernel

// 1 over a power of two from 2^-126 to 2^126.
SLS_DEV float q8_inverse(float x) { return __int_as_float(0x7f000000 - __float_as_int(x)); }
// The least power of two from 2^-126 to 2^126 that is at least x.
SLS_DEV float q8_power(float x) {
  const int bits = __float_as_int(x), e = (bits >> 23) + ((bits & 0x7fffff) != 0);
  return __int_as_float(min(max(e, 1), 253) << 23);
}
// The unit of a head's weights (times values' scales) from this step on, a power of two.  None of
// them may be larger; a much larger unit costs their float16 bits, and all of them past 2^39.  So it
// goes by what a step needs, most = its largest weight times scale, and not by its scales alone: tokens
// that the head does not look at may have any (2^40 times the others' made its results zeros).  Within
// 16 of that it takes the step's largest scale all the same, and rises seldom: a unit is less than 32
// times what is needed.  was: the unit before, shrink: what the earlier weights are multiplied by now.
// The unit stays within 2^126 of the step's scales, so that no scale in units overflows.
SLS_DEV float q8_unit(float was, float shrink, float scale, float most) {
  float u = fmaxf(was * shrink, fminf(was, most));
  if (scale > u) u = scale <= 16.f * most ? scale : fmaxf(fmaxf(u, most), scale * 0x1p-126f);
  return q8_power(u);
}

// NH: blocks of eight query heads a key head
template <int HD, int NH>
struct Q8Shape {
  static constexpr int WARPS = NH == 1 ? 12 : 8;
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int VB = HD / 8;               // bytes of a value that a lane reads
  static constexpr int CHUNKS = HD / 64;          // 16-byte reads of a key for each of four lanes
  static constexpr int MAT_BYTES = AD_KEYS * HD;  // keys or values of a step
  static constexpr int STAGE_BYTES = 2 * MAT_BYTES;
  static constexpr int STAGES = (NH == 1 ? 2 : 3) * 128 / HD;
  static constexpr size_t SMEM = (size_t)WARPS * STAGES * STAGE_BYTES + 1024;
  // Byte of 16-byte chunk ch of row `key` of keys or values, as the copies' swizzle left it.
  SLS_DEV static int at(int key, int ch) {
    return HD == 128 ? key * 128 + ((ch ^ (key & 7)) << 4) : key * 64 + ((ch ^ (key >> 1 & 3)) << 4);
  }
};

SLS_DEV uint32_t q8_transpose(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A warp's ring: its next steps are copied ahead, from sequence to sequence.  Codes come by TMA,
// counted by a barrier; scales, a float for each half of a step, by cp.async, one group a step.
template <int HD, int NH>
struct Q8Ring {
  using S = Q8Shape<HD, NH>;
  const CacheView& c;
  const ScaleView& sc;
  const CUtensorMap* tmK;
  const CUtensorMap* tmV;
  unsigned char* mem;
  uint64_t* bars;
  float4* scales;    // of each stage: keys' and values' scales of its two halves
  int* status;
  int kvh;
  uint32_t lead;
  int is, ij, ilen;  // the step to issue next: its sequence, its number there, the length
  int64_t left;      // steps still to issue
  int batch0, page;  // lane l: the page of tokens 16 l of the batch of 16 steps from batch0 on
  unsigned issued, used;

  SLS_DEV Q8Ring(const CacheView& cache, const ScaleView& s, const CUtensorMap* k,
                 const CUtensorMap* v, unsigned char* ring, uint64_t* b, float4* f, int* word,
                 int head, int seq, int step, int len, int64_t n)
      : c(cache), sc(s), tmK(k), tmV(v), mem(ring), bars(b), scales(f), status(word), kvh(head),
        lead(at_elect()), is(seq), ij(step), ilen(len), left(n), batch0(-1), page(-1), issued(0),
        used(0) {
#pragma unroll 1
    for (int i = 0; i < S::STAGES; ++i) issue();
  }

  SLS_DEV void issue() {
    if (left > 0) {
      if (ij * AD_KEYS >= ilen) {
        do {
          ++is;
          ilen = (int)cache_len(c, is);
        } while (ilen == 0);
        ij = 0;
        batch0 = -1;
      }
      const int lane = threadIdx.x & 31;
      if (batch0 < 0 || ij - batch0 == 16) {
        batch0 = ij;
        const int x = ij * AD_KEYS + 16 * lane;
        page = x < ilen ? c.table[is * c.table_ld + (x >> c.page_shift)] : -1;
      }
      const unsigned st = issued % S::STAGES;
      const int box = min(AD_KEYS, 1 << c.page_shift);  // 16 or 32 slots of one copy
      const int copies = (min(AD_KEYS, ilen - ij * AD_KEYS) + box - 1) / box;
      const int slot0 = (ij * AD_KEYS) & ((1 << c.page_shift) - 1);
      if (lead) mbar_expect_tx(&bars[st], 2 * copies * box * HD);
      __syncwarp();
      const int first = 2 * (ij - batch0);
#pragma unroll 1
      for (int cp = 0; cp < copies; ++cp) {
        const int pg = __shfl_sync(0xffffffffu, page, first + cp);
        const uint32_t dst = smem_u32(mem) + st * S::STAGE_BYTES + cp * box * HD;
        at_tma4(lead, dst, tmK, 0, slot0, kvh, pg, &bars[st]);
        at_tma4(lead, dst + S::MAT_BYTES, tmV, 0, slot0, kvh, pg, &bars[st]);
      }
      // lanes 0, 1: keys' scales of tokens 0 .. 15 and 16 .. 31; 2, 3: values'
      const int g = lane & 1;
      const int64_t pg = __shfl_sync(0xffffffffu, page, first + g);
      if (lane < 4) {
        const int slot = (ij * AD_KEYS + 16 * g) & ((1 << c.page_shift) - 1);
        const bool real = ij * AD_KEYS + 16 * g < ilen && pg >= 0 && pg < c.num_pages;
        const float* f = lane < 2 ? sc.k : sc.v;
        if (real) f += pg * sc.page + (slot >> sc.shift) * sc.block + kvh * sc.head;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(
                         smem_u32(scales + st) + 4 * lane),
                     "l"(f), "r"(real ? 4 : 0)
                     : "memory");
      }
      ++ij;
      ++issued;
      --left;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  // Waits for the next step; false when the time is up, after the other copies in
  // flight have landed or run out of time too.
  SLS_DEV bool wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
    if (__all_sync(0xffffffffu, mbar_wait(&bars[used % S::STAGES], (used / S::STAGES) & 1)))
      return true;
    if ((threadIdx.x & 31) == 0) atomicExch(status, SLS_ERR_TIMEOUT);
    for (unsigned x = used + 1; x < issued; ++x)
      mbar_wait(&bars[x % S::STAGES], (x / S::STAGES) & 1);
    return false;
  }
};

// The rows of a piece: queries as operands (lane / 4: the head), unnormalised outputs (VB elements of
// heads 2 (lane % 4) and the next), those heads' maxima in use, this lane's part of their sums of
// weights, and 1 over the units that outputs are in.
template <typename E, typename C, int HD, int NH>
struct Q8Rows {
  using S = Q8Shape<HD, NH>;
  static constexpr int KS = HD / 16;  // 16-element slices of a head
  static constexpr int MT = HD / 16;  // 16-row tiles of outputs
  uint32_t q[NH][KS][2];
  float o[NH][MT][4];
  float mx[NH][2], l[NH][2], qf[NH][2], per[NH][2];

  SLS_DEV void start(const AttnArgs& a, int seq, int head0, int rows) {
    const int lane = threadIdx.x & 31, r = lane >> 2, cq = lane & 3;
    const char* qp = a.q.data + seq * a.q.token_b + head0 * a.q.head_b;
#pragma unroll
    for (int x = 0; x < NH; ++x) {
      const int rr = r + 8 * x;
      uint2 raw[KS];
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int e = 64 * (k >> 2) + 16 * cq + 4 * (k & 3);
        raw[k] = (rr < rows && e < a.c.head_dim)
                     ? *reinterpret_cast<const uint2*>(qp + rr * a.q.head_b + 2 * e)
                     : make_uint2(0u, 0u);
        const float2 f = Half2<E>::widen(raw[k].x), g = Half2<E>::widen(raw[k].y);
        top = fmaxf(fmaxf(fmaxf(top, fabsf(f.x)), fmaxf(fabsf(f.y), fabsf(g.x))), fabsf(g.y));
      }
      float back = 1.f;
      if constexpr (std::is_same<E, __half>::value) {
#pragma unroll
        for (int k = 0; k < KS; ++k) q[x][k][0] = raw[k].x, q[x][k][1] = raw[k].y;
      } else {
        // the largest element to [2^14, 2^15)
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = max(__float_as_int(top) >> 23, 16);
        const float by = __int_as_float((127 + 14 + 127 - e) << 23);
        back = __int_as_float((e - 14) << 23);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const float2 f = Half2<E>::widen(raw[k].x), g = Half2<E>::widen(raw[k].y);
          q[x][k][0] = Half2<__half>::narrow(f.x * by, f.y * by);
          q[x][k][1] = Half2<__half>::narrow(g.x * by, g.y * by);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        qf[x][j] = __shfl_sync(0xffffffffu, back, 4 * (2 * cq + j));
        mx[x][j] = -INFINITY;
        l[x][j] = 0.f;
        per[x][j] = 0x1p126f;
      }
#pragma unroll
      for (int b = 0; b < MT; ++b) o[x][b][0] = o[x][b][1] = o[x][b][2] = o[x][b][3] = 0.f;
    }
  }

  // steps [j0, j1) of a sequence of `len` tokens; cs: scale log2(e)
  SLS_DEV bool run(Q8Ring<HD, NH>& ring, int len, int j0, int j1, float cs) {
    const int lane = threadIdx.x & 31, r = lane >> 2, cq = lane & 3;
    const int mine = ad_token(r);  // the token of this lane's rows r and (8 more) r + 8
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
      if (!ring.wait()) return false;
      __syncwarp();  // the scales are copied by lanes 0 to 3
      const unsigned st = ring.used % S::STAGES;
      const unsigned char* stage = ring.mem + st * S::STAGE_BYTES;
      const float4 f4 = ring.scales[st];
      const int lim = len - j * AD_KEYS;
      float s[NH][2][4];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
        for (int x = 0; x < NH; ++x) s[x][mt][0] = s[x][mt][1] = s[x][mt][2] = s[x][mt][3] = 0.f;
#pragma unroll
        for (int i = 0; i < S::CHUNKS; ++i) {
          const int key = 16 * mt + mine;
          const uint4 u = *reinterpret_cast<const uint4*>(stage + S::at(key, 4 * i + cq));
          const uint4 v = *reinterpret_cast<const uint4*>(stage + S::at(key + 8, 4 * i + cq));
          const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            uint32_t k[4];
            codes_half<C>(uw[y], k[0], k[2]);
            codes_half<C>(vw[y], k[1], k[3]);
#pragma unroll
            for (int x = 0; x < NH; ++x)
              mma16816<__half>(s[x][mt], k, q[x][4 * i + y][0], q[x][4 * i + y][1]);
          }
        }
      }
      // true scores: powers of two, so exactly (scales of the caller's own: to one rounding)
#pragma unroll
      for (int x = 0; x < NH; ++x) {
        const float k0 = f4.x * qf[x][0], k1 = f4.x * qf[x][1], k2 = f4.y * qf[x][0],
                    k3 = f4.y * qf[x][1];
        s[x][0][0] *= k0, s[x][0][1] *= k1, s[x][0][2] *= k0, s[x][0][3] *= k1;
        s[x][1][0] *= k2, s[x][1][1] *= k3, s[x][1][2] *= k2, s[x][1][3] *= k3;
      }
      if (lim < AD_KEYS) {
#pragma unroll
        for (int x = 0; x < NH; ++x)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (16 * mt + mine + 8 * (i >> 1) >= lim) s[x][mt][i] = -INFINITY;
      }
      float top[NH][2];
      bool up = false;
      const float vmax = fmaxf(fabsf(f4.z), fabsf(f4.w));
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m = fmaxf(fmaxf(s[x][0][i], s[x][0][2 + i]), fmaxf(s[x][1][i], s[x][1][2 + i]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
          top[x][i] = fmaxf(m, mx[x][i]);
          up |= top[x][i] > mx[x][i] || vmax * per[x][i] > 1.f;
        }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int x = 0; x < NH; ++x) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            // the halves' largest weights
            float most[2];
            const float base = top[x][i] == -INFINITY ? 0.f : top[x][i];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              float m = fmaxf(s[x][mt][i], s[x][mt][2 + i]);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
              most[mt] = at_exp2((m - base) * cs);
            }
            f[i] = top[x][i] > mx[x][i] ? at_exp2((mx[x][i] - top[x][i]) * cs) : 1.f;
            mx[x][i] = top[x][i];
            l[x][i] *= f[i];
            const float was = q8_inverse(per[x][i]);
            per[x][i] = q8_inverse(
                q8_unit(was, f[i], vmax, fmaxf(most[0] * fabsf(f4.z), most[1] * fabsf(f4.w))));
            f[i] = f[i] * was * per[x][i];
          }
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            o[x][b][0] *= f[0], o[x][b][1] *= f[1];
            o[x][b][2] *= f[0], o[x][b][3] *= f[1];
          }
        }
      }
      uint32_t w[NH][2][2];
#pragma unroll
      for (int x = 0; x < NH; ++x) {
        // the distance from the maximum first, as in the 16-bit kernel
        const float base[2] = {mx[x][0] == -INFINITY ? 0.f : mx[x][0],
                               mx[x][1] == -INFINITY ? 0.f : mx[x][1]};
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const float vs[2] = {(mt ? f4.w : f4.z) * per[x][0], (mt ? f4.w : f4.z) * per[x][1]};
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = at_exp2(__fmaf_rn(s[x][mt][i] - base[i & 1], cs, Q8_SHIFT));
            sum[i & 1] += e[i];
            e[i] *= vs[i & 1];
          }
          w[x][mt][0] = q8_transpose(Half2<__half>::narrow(e[0], e[1]));
          w[x][mt][1] = q8_transpose(Half2<__half>::narrow(e[2], e[3]));
        }
        l[x][0] += sum[0], l[x][1] += sum[1];
      }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint32_t v[4][S::VB / 4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int key = 16 * mt + ad_token(2 * cq + (y & 1)) + 8 * (y >> 1);
          const unsigned char* p = stage + S::MAT_BYTES;
          if constexpr (S::VB == 16) {
            uint4 u = *reinterpret_cast<const uint4*>(p + S::at(key, r));
            if (key >= lim) u = make_uint4(0, 0, 0, 0);  // past the end: whatever its slot holds
            v[y][0] = u.x, v[y][1] = u.y, v[y][2] = u.z, v[y][3] = u.w;
          } else {
            uint2 u = *reinterpret_cast<const uint2*>(p + S::at(key, r >> 1) + 8 * (r & 1));
            if (key >= lim) u = make_uint2(0, 0);
            v[y][0] = u.x, v[y][1] = u.y;
          }
        }
#pragma unroll
        for (int y = 0; y < S::VB / 4; ++y) {
          uint32_t f[2][4];
          codes_half<C>(__byte_perm(v[0][y], v[1][y], 0x5140), f[0][0], f[0][1]);
          codes_half<C>(__byte_perm(v[0][y], v[1][y], 0x7362), f[1][0], f[1][1]);
          codes_half<C>(__byte_perm(v[2][y], v[3][y], 0x5140), f[0][2], f[0][3]);
          codes_half<C>(__byte_perm(v[2][y], v[3][y], 0x7362), f[1][2], f[1][3]);
#pragma unroll
          for (int x = 0; x < NH; ++x) {
            mma16816<__half>(o[x][2 * y], f[0], w[x][mt][0], w[x][mt][1]);
            mma16816<__half>(o[x][2 * y + 1], f[1], w[x][mt][0], w[x][mt][1]);
          }
        }
      }
      __syncwarp();
      ++ring.used;
      ring.issue();
    }
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[x][i] += __shfl_xor_sync(0xffffffffu, l[x][i], d);
    return true;
  }

  // element e of this lane's VB of head 2 (lane % 4) + i of block x
  SLS_DEV float out(int x, int i, int e) const { return o[x][e >> 1][2 * (e & 1) + i]; }
};

template <typename E, typename C, int HD, int NH>
__global__ void __launch_bounds__(Q8Shape<HD, NH>::THREADS, 1)
attention_decode_q8_kernel(const __grid_constant__ CUtensorMap tmK,
                           const __grid_constant__ CUtensorMap tmV,
                           const __grid_constant__ AttnArgs a, const __grid_constant__ ScaleView sc,
                           const __grid_constant__ AdPlan p, int* status) {
  using S = Q8Shape<HD, NH>;
  constexpr int AD_T = S::THREADS;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ int64_t s_pre[AD_T + 1];
  __shared__ float4 s_scale[S::WARPS][S::STAGES];
  __shared__ uint64_t full_bar[S::WARPS][S::STAGES];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  at_wait_ahead();
  if (lane < S::STAGES) mbar_init(&full_bar[warp][lane], 1);
  mbar_fence_init();
  const auto steps = [&](int s) { return ad_steps(c, s); };
  const int R = ad_prefix<AD_T>(c, s_pre, p.prefix, steps);
  const int64_t total = s_pre[AD_T];
  const int parts = ad_parts(total, p.groups);
  const int gw = blockIdx.x * S::WARPS + warp;
  const int g = gw / p.vheads, vh = gw - g * p.vheads;
  if (g >= parts) return;
  const int64_t t0 = ad_div(total * g, parts), t1 = ad_div(total * (g + 1), parts);
  const int group = a.q_heads / c.kv_heads;
  const int blocks = (group + AD_ROWS - 1) / AD_ROWS;
  const int kvh = vh / blocks, row0 = (vh - kvh * blocks) * AD_ROWS;
  const int rows = min(AD_ROWS, group - row0);
  const int head0 = kvh * group + row0;
  int seq;
  int64_t before;  // steps before seq
  ad_find<AD_T>(s_pre, R, t0, steps, seq, before);

  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Q8Ring<HD, NH> ring(c, sc, &tmK, &tmV, smem + warp * S::STAGES * S::STAGE_BYTES, full_bar[warp],
                      s_scale[warp], status, kvh, seq, (int)(t0 - before), (int)cache_len(c, seq),
                      t1 - t0);
  const float cs = a.scale * 1.4426950408889634f;
  const int e0 = S::VB * (lane >> 2);
  int64_t t = t0;
  while (t < t1) {
    // ---- a piece: steps [j0, j1) of sequence seq ----
    const int len = (int)cache_len(c, seq);
    const int n = (len + AD_KEYS - 1) / AD_KEYS;
    if (n == 0) {
      ++seq;
      continue;
    }
    const int j0 = (int)(t - before);
    const int j1 = (int)min((int64_t)n, t1 - before);
    Q8Rows<E, C, HD, NH> w;
    w.start(a, seq, head0, rows);
    if (!w.run(ring, len, j0, j1, cs)) return;
    const bool whole = j0 == 0 && j1 == n;
    // the part's first piece goes to slot 0, a later one (its last) to slot 1
    const int64_t slot = ((int64_t)(2 * g + (t > t0)) * p.vheads + vh) * AD_ROWS;
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int rr = 8 * x + 2 * (lane & 3) + i;
        if (rr >= rows) continue;
        if (!whole && lane < 4) p.ml[slot + rr] = make_float2(w.mx[x][i], w.l[x][i]);
        if (e0 >= c.head_dim) continue;
        const float unit = q8_inverse(w.per[x][i]), f = whole ? 1.f / w.l[x][i] : 1.f;
        char* out = a.out.data + seq * a.out.token_b + (head0 + rr) * a.out.head_b + 2 * e0;
        float* piece = p.o + (slot + rr) * p.hd_pad + e0;
#pragma unroll
        for (int b = 0; b < S::VB; b += 8) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = w.out(x, i, b + k) * f * unit;
          if (whole) {
            *reinterpret_cast<uint4*>(out + 2 * b) = narrow8<E>(y);
          } else {
            *reinterpret_cast<float4*>(piece + b) = make_float4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<float4*>(piece + b + 4) = make_float4(y[4], y[5], y[6], y[7]);
          }
        }
      }
    t = before + j1;
    if (j1 == n) {
      before += n;
      ++seq;
    }
  }
}

// Few rows: a cluster of CTAs owns a (sequence, key head); pieces meet in shared memory and are
// joined there, as in the 16-bit kernel: one launch, no workspace.
template <typename E, typename C, int HD, int NH>
__global__ void __launch_bounds__(Q8Shape<HD, NH>::THREADS, 1)
attention_decode_q8_cluster_kernel(const __grid_constant__ CUtensorMap tmK,
                                   const __grid_constant__ CUtensorMap tmV,
                                   const __grid_constant__ AttnArgs a,
                                   const __grid_constant__ ScaleView sc, int vheads, int* status) {
  using S = Q8Shape<HD, NH>;
  constexpr int W = S::WARPS, ROWS = 8 * NH;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t full_bar[W][S::STAGES];
  __shared__ float4 s_scale[W][S::STAGES];
  __shared__ float s_m[W][ROWS], s_l[W][ROWS];
  __shared__ float s_join[W][HD + 2];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int unit = blockIdx.x / size;
  const int seq = unit / vheads, kvh = unit - seq * vheads;
  const int rows = a.q_heads / c.kv_heads, head0 = kvh * rows;
  if (lane < S::STAGES) mbar_init(&full_bar[warp][lane], 1);
  mbar_fence_init();
  __syncwarp();
  at_go();
  at_wait_ahead();

  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* mine = smem + warp * S::STAGES * S::STAGE_BYTES;
  const int len = (int)cache_len(c, seq);
  const int n = (len + AD_KEYS - 1) / AD_KEYS;
  const int me = rank * W + warp, all = size * W;
  const int j0 = (int)((int64_t)n * me / all), j1 = (int)((int64_t)n * (me + 1) / all);
  Q8Ring<HD, NH> ring(c, sc, &tmK, &tmV, mine, full_bar[warp], s_scale[warp], status, kvh, seq, j0,
                      len, j1 - j0);
  Q8Rows<E, C, HD, NH> w;
  w.start(a, seq, head0, rows);
  const float cs = a.scale * 1.4426950408889634f;
  const bool ok = w.run(ring, len, j0, j1, cs);
  // the outputs go where the warp's ring was
  static_assert(S::STAGES * S::STAGE_BYTES >= ROWS * HD * 4, "a ring holds a piece");
  float* out_s = reinterpret_cast<float*>(mine);
  __syncwarp();
#pragma unroll
  for (int x = 0; x < NH; ++x)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int rr = 8 * x + 2 * (lane & 3) + i;
      if (lane < 4) {
        s_m[warp][rr] = w.mx[x][i];
        s_l[warp][rr] = ok ? w.l[x][i] : 0.f;
      }
      if (rr >= rows) continue;
      const float unit = q8_inverse(w.per[x][i]);
#pragma unroll
      for (int b = 0; b < S::VB; b += 4)
        *reinterpret_cast<float4*>(out_s + rr * HD + S::VB * (lane >> 2) + b) =
            make_float4(w.out(x, i, b) * unit, w.out(x, i, b + 1) * unit,
                        w.out(x, i, b + 2) * unit, w.out(x, i, b + 3) * unit);
    }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  ad_cluster_join<E, HD, W>(a, seq, head0, rows, n, rank, size, cs, s_m[0], s_l[0], ROWS, out_s,
                            s_join);
  // no CTA leaves while another reads its shared memory
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename E, typename C, int HD, int NH>
int launch(const AttnArgs& a, const ScaleView& s, const AdHost& h, void* workspace,
           cudaStream_t stream) {
  using S = Q8Shape<HD, NH>;
  static bool set[64] = {};  // per device
  static int* words[64] = {};
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto parts = attention_decode_q8_kernel<E, C, HD, NH>;
  auto cluster = attention_decode_q8_cluster_kernel<E, C, HD, NH>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(parts, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)S::SMEM));
    SLS_CUDA_TRY(cudaFuncSetAttribute(cluster, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)S::SMEM));
  }
  int* word = dev < 64 ? words[dev] : nullptr;
  if (!word) {
    const int st = decode_status_word(&word);
    if (st != SLS_OK) return st;
  }
  if (dev < 64) words[dev] = word, set[dev] = true;
  const CacheView& c = a.c;
  CUtensorMap k, v;
  const int slots = std::min(AD_KEYS, 1 << c.page_shift);
  if (!at_code_map<HD>(&k, c, c.k, slots) || !at_code_map<HD>(&v, c, c.v, slots))
    return SLS_ERR_UNSUPPORTED;
  if (h.cluster > 0)
    return at_launch(cluster, dim3((unsigned)(c.B * h.vheads * h.cluster)), S::THREADS, S::SMEM,
                     h.cluster, stream, k, v, a, s, h.vheads, word);
  const AdPlan p = ad_plan(h, workspace);
  const int st = at_launch(parts, dim3((unsigned)h.grid), S::THREADS, S::SMEM, 1, stream, k, v, a,
                           s, p, word);
  if (st != SLS_OK) return st;
  return ad_join<E>(a, p, stream);
}

template <typename E, typename C>
int launch(const AttnArgs& a, const ScaleView& s, const AdHost& h, void* workspace,
           cudaStream_t stream) {
  const bool eight = a.q_heads / a.c.kv_heads <= 8;
  if (a.c.head_dim > 64)
    return eight ? launch<E, C, 128, 1>(a, s, h, workspace, stream)
                 : launch<E, C, 128, 2>(a, s, h, workspace, stream);
  return eight ? launch<E, C, 64, 1>(a, s, h, workspace, stream)
               : launch<E, C, 64, 2>(a, s, h, workspace, stream);
}

int q8_host(const CacheView& c, int q_heads, AdHost* h) {
  const bool eight = q_heads / c.kv_heads <= 8;
  return ad_host(c, q_heads, eight ? Q8Shape<128, 1>::WARPS : Q8Shape<128, 2>::WARPS, h);
}

}  // namespace

size_t attention_decode_q8_workspace(const CacheView& c, int q_heads) {
  AdHost h;
  if (c.B == 0 || q8_host(c, q_heads, &h) != SLS_OK || h.cluster > 0) return 0;
  return h.prefix_b + h.ml_b + h.o_b;
}

int launch_attention_decode_q8(const AttnArgs& a, const ScaleView& s, int code, int dtype,
                               void* workspace, cudaStream_t stream) {
  if (a.c.B == 0) return SLS_OK;
  if ((int64_t)a.c.B * a.q_heads > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  AdHost h;
  const int st = q8_host(a.c, a.q_heads, &h);
  if (st != SLS_OK) return st;
  if (dtype == SLS_BF16)
    return code == SLS_I8 ? launch<__nv_bfloat16, I8>(a, s, h, workspace, stream)
                          : launch<__nv_bfloat16, E4M3>(a, s, h, workspace, stream);
  return code == SLS_I8 ? launch<__half, I8>(a, s, h, workspace, stream)
                        : launch<__half, E4M3>(a, s, h, workspace, stream);
}

}  // namespace sls
