// One new token per sequence over a paged cache of 8-bit codes: o = softmax(scale q K^T) V with
// k = sk c^k and v = sv c^v, codes and scales read once.
//
// Bound by HBM bandwidth: 2 hd bytes a cached token and key head.  A warp owns a (sequence,
// key head) at a time, its rows and pieces as in the 16-bit kernel, and multiplies float16
// (every code is one exactly) by mma.sync.  What the 8 bits change:
//  * The scale of a block of tokens multiplies finished scores, and weights instead of values
//    (in units of the largest value scale so far, so that they stay in float16's range).
//  * bfloat16 queries become float16 times a power of two for each row, which scores take back:
//    exact unless an element is below 2^-38 of its row's largest.
//  * A fragment of keys is sixteen consecutive bytes of one key, the elements of a head taken in
//    an order of their own (the same for queries); a fragment of values is sixteen bytes of four
//    keys, bytes of two keys interleaved on the way to float16.  So a lane needs only bytes that
//    it can copy itself: it fetches them by cp.async into shared memory that no other lane
//    reads, `STAGES` steps of 32 tokens ahead, and no barrier or transposing load follows.
#include <algorithm>

#include "attention_decode.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr float Q8_SHIFT = 15.f;  // log2 of a factor of all weights, see the 16-bit kernel

template <int HD>
struct Q8Shape {
  static constexpr int WARPS = 8;
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int VB = HD / 8;                      // bytes of a key that a lane's copy of values has
  static constexpr int CHUNKS = HD / 64;                 // 16-byte copies of a key for its four lanes
  static constexpr int MAT_BYTES = AD_KEYS * HD;         // keys or values of a step
  static constexpr int STAGE_BYTES = 2 * MAT_BYTES;
  static constexpr int STAGES = HD == 128 ? 3 : 6;
  static constexpr size_t SMEM = (size_t)WARPS * STAGES * STAGE_BYTES;
};

// `bytes` (0 or all) of the copy are read, the rest is zero.
template <int N>
SLS_DEV void q8_copy(uint32_t dst, const char* src, bool read) {
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
                 "r"(read ? 16 : 0)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N),
                 "r"(read ? N : 0)
                 : "memory");
}
SLS_DEV void q8_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
SLS_DEV void q8_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A warp's ring: its next steps are copied ahead, from sequence to sequence.  One group of
// copies a step, empty ones past the last, so that STAGES - 1 are in flight behind the oldest.
template <int HD>
struct Q8Ring {
  using S = Q8Shape<HD>;
  const CacheView& c;
  const ScaleView& sc;
  unsigned char* mem;
  float4* scales;    // of each stage: keys' and values' scales of its two halves
  int kvh;
  int is, ij, ilen;  // the step to issue next: its sequence, its number there, the length
  int64_t left;      // steps still to issue
  int batch0, page;  // lane l: the page of tokens 16 l of the batch of 16 steps from batch0 on
  unsigned st_in, st_out;

  SLS_DEV Q8Ring(const CacheView& cache, const ScaleView& s, unsigned char* ring, float4* f,
                 int head, int seq, int step, int len, int64_t n)
      : c(cache), sc(s), mem(ring), scales(f), kvh(head), is(seq), ij(step), ilen(len), left(n),
        batch0(-1), page(-1), st_in(0), st_out(0) {
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
      const int lane = threadIdx.x & 31, n = lane >> 2, q = lane & 3;
      if (batch0 < 0 || ij - batch0 == 16) {
        batch0 = ij;
        const int x = ij * AD_KEYS + 16 * lane;
        page = x < ilen ? c.table[is * c.table_ld + (x >> c.page_shift)] : -1;
        if ((unsigned)page >= (uint64_t)c.num_pages) page = -1;
      }
      const int lim = ilen - ij * AD_KEYS;  // tokens from the step's first on
      const uint32_t dst = smem_u32(mem) + st_in * S::STAGE_BYTES;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int pg = __shfl_sync(0xffffffffu, page, 2 * (ij - batch0) + g);
        const int slot = (ij * AD_KEYS + 16 * g) & ((1 << c.page_shift) - 1);
        const int64_t at = max(pg, 0) * c.page_b + slot * c.slot_b + kvh * c.head_b;
        const int lim_g = pg < 0 ? 0 : lim - 16 * g;
        const char* k = c.k + at + n * c.slot_b + 16 * q;
        const char* v = c.v + at + 2 * q * c.slot_b + S::VB * n;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < S::CHUNKS; ++i) {
            const bool on = 64 * i + 16 * q < c.head_dim && 8 * b + n < lim_g;
            q8_copy<16>(dst + ((2 * g + b) * S::CHUNKS + i) * 512 + 16 * lane,
                        on ? k + 8 * b * c.slot_b + 64 * i : c.k, on);
          }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int key = (x & 1) + 8 * (x >> 1);
          const bool on = S::VB * n < c.head_dim && 2 * q + key < lim_g;
          q8_copy<S::VB>(dst + S::MAT_BYTES + (4 * g + x) * 32 * S::VB + S::VB * lane,
                         on ? v + key * c.slot_b : c.v, on);
        }
        if (lane < 2) {
          const float* f = lane == 0 ? sc.k : sc.v;
          if (lim_g > 0) f += pg * sc.page + (slot >> sc.shift) * sc.block + kvh * sc.head;
          q8_copy<4>(smem_u32(scales + st_in) + 8 * lane + 4 * g,
                     reinterpret_cast<const char*>(f), lim_g > 0);
        }
      }
      ++ij;
      --left;
    }
    q8_commit();
    st_in = st_in + 1 == S::STAGES ? 0 : st_in + 1;
  }
};

// The rows of a piece: queries as A fragments, unnormalised outputs in units of sv, the maximum
// in use and this lane's part of the sum of weights, for rows lane / 4 and lane / 4 + 8.
template <typename E, typename C, int HD>
struct Q8Rows {
  using S = Q8Shape<HD>;
  static constexpr int KS = HD / 16;  // 16-element slices of a head
  static constexpr int NT = HD / 8;   // columns of outputs: element VB n + t for lane group n
  uint32_t q[KS][4];
  float o[NT][4];
  float mx[2], l[2], qf[2];
  float sv;

  SLS_DEV void start(const AttnArgs& a, int seq, int head0, int rows) {
    const int lane = threadIdx.x & 31, r = lane >> 2, cq = lane & 3;
    const char* qp = a.q.data + seq * a.q.token_b + head0 * a.q.head_b;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
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
      qf[x] = 1.f;
      if constexpr (std::is_same<E, __half>::value) {
#pragma unroll
        for (int k = 0; k < KS; ++k) q[k][x] = raw[k].x, q[k][2 + x] = raw[k].y;
      } else {
        // the largest element to [2^14, 2^15)
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = max(__float_as_int(top) >> 23, 16);
        const float by = __int_as_float((127 + 14 + 127 - e) << 23);
        qf[x] = __int_as_float((e - 14) << 23);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const float2 f = Half2<E>::widen(raw[k].x), g = Half2<E>::widen(raw[k].y);
          q[k][x] = Half2<__half>::narrow(f.x * by, f.y * by);
          q[k][2 + x] = Half2<__half>::narrow(g.x * by, g.y * by);
        }
      }
    }
#pragma unroll
    for (int b = 0; b < NT; ++b) o[b][0] = o[b][1] = o[b][2] = o[b][3] = 0.f;
    mx[0] = mx[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    sv = 0.f;
  }

  // steps [j0, j1) of a sequence of `len` tokens; cs: scale log2(e)
  SLS_DEV void run(Q8Ring<HD>& ring, int len, int j0, int j1, float cs) {
    const int lane = threadIdx.x & 31, cq = 2 * (lane & 3);
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
      q8_wait<S::STAGES - 1>();
      __syncwarp();  // the scales are copied by lanes 0 and 1
      const unsigned char* stage = ring.mem + ring.st_out * S::STAGE_BYTES;
      const float4 f4 = ring.scales[ring.st_out];
      const int lim = len - j * AD_KEYS;
      float s[4][4];
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
#pragma unroll
        for (int i = 0; i < S::CHUNKS; ++i) {
          const uint4 k = *reinterpret_cast<const uint4*>(stage + (nb * S::CHUNKS + i) * 512 +
                                                          16 * lane);
          const uint32_t w[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t b0, b1;
            codes_half<C>(w[x], b0, b1);
            mma16816<__half>(s[nb], q[4 * i + x], b0, b1);
          }
        }
      }
      // true scores: powers of two, so exactly (scales of the caller's own: to one rounding)
      const float ks[2][2] = {{f4.x * qf[0], f4.x * qf[1]}, {f4.y * qf[0], f4.y * qf[1]}};
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nb][i] *= ks[nb >> 1][i >> 1];
      if (lim < AD_KEYS) {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (nb * 8 + cq + (i & 1) >= lim) s[nb][i] = -INFINITY;
      }
      float top[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float m = fmaxf(s[0][2 * x], s[0][2 * x + 1]);
#pragma unroll
        for (int nb = 1; nb < 4; ++nb) m = fmaxf(fmaxf(m, s[nb][2 * x]), s[nb][2 * x + 1]);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        top[x] = fmaxf(m, mx[x]);
      }
      const float nsv = fmaxf(sv, fmaxf(f4.z, f4.w));
      if (__any_sync(0xffffffffu, top[0] > mx[0] || top[1] > mx[1]) || nsv > sv) {
        const float g = nsv > sv ? sv / nsv : 1.f;
        float f[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          f[x] = top[x] > mx[x] ? at_exp2((mx[x] - top[x]) * cs) : 1.f;
          mx[x] = top[x];
          l[x] *= f[x];
          f[x] *= g;
        }
        sv = nsv;
#pragma unroll
        for (int b = 0; b < NT; ++b) {
          o[b][0] *= f[0], o[b][1] *= f[0];
          o[b][2] *= f[1], o[b][3] *= f[1];
        }
      }
      const float unit = sv > 0.f ? 1.f / sv : 0.f;
      const float vs[2] = {f4.z * unit, f4.w * unit};
      // the distance from the maximum first, as in the 16-bit kernel
      const float base[2] = {mx[0] == -INFINITY ? 0.f : mx[0], mx[1] == -INFINITY ? 0.f : mx[1]};
      uint32_t w[2][4];
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[i] = at_exp2(__fmaf_rn(s[nb][i] - base[i >> 1], cs, Q8_SHIFT));
          sum[i >> 1] += e[i];
          e[i] *= vs[nb >> 1];
        }
        w[nb >> 1][2 * (nb & 1)] = Half2<__half>::narrow(e[0], e[1]);
        w[nb >> 1][2 * (nb & 1) + 1] = Half2<__half>::narrow(e[2], e[3]);
      }
      l[0] += sum[0], l[1] += sum[1];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t v[4][S::VB / 4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const unsigned char* p = stage + S::MAT_BYTES + (4 * g + x) * 32 * S::VB + S::VB * lane;
          if constexpr (S::VB == 16) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            v[x][0] = u.x, v[x][1] = u.y, v[x][2] = u.z, v[x][3] = u.w;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            v[x][0] = u.x, v[x][1] = u.y;
          }
        }
#pragma unroll
        for (int y = 0; y < S::VB / 4; ++y) {
          uint32_t b0[4], b1[4];
          codes_half<C>(__byte_perm(v[0][y], v[1][y], 0x5140), b0[0], b0[1]);
          codes_half<C>(__byte_perm(v[0][y], v[1][y], 0x7362), b0[2], b0[3]);
          codes_half<C>(__byte_perm(v[2][y], v[3][y], 0x5140), b1[0], b1[1]);
          codes_half<C>(__byte_perm(v[2][y], v[3][y], 0x7362), b1[2], b1[3]);
#pragma unroll
          for (int x = 0; x < 4; ++x) mma16816<__half>(o[4 * y + x], w[g], b0[x], b1[x]);
        }
      }
      __syncwarp();
      ring.st_out = ring.st_out + 1 == S::STAGES ? 0 : ring.st_out + 1;
      ring.issue();
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
    }
  }

  // first of the VB elements from o[0 ..][2 x + cc] on
  SLS_DEV static int element(int cc) { return S::VB * (2 * (threadIdx.x & 3) + cc); }
};

template <typename E, typename C, int HD>
__global__ void __launch_bounds__(Q8Shape<HD>::THREADS, 1)
attention_decode_q8_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ ScaleView sc,
                           const __grid_constant__ AdPlan p) {
  using S = Q8Shape<HD>;
  constexpr int AD_T = S::THREADS;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int64_t s_pre[AD_T + 1];
  __shared__ float4 s_scale[S::WARPS][S::STAGES];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  at_wait_ahead();
  const int R = ad_prefix<AD_T>(c, s_pre, p.prefix);
  const int64_t total = s_pre[AD_T];
  const int parts = ad_parts(total, p.groups);
  const int gw = blockIdx.x * S::WARPS + warp;
  const int g = gw / p.vheads, vh = gw - g * p.vheads;
  if (g >= parts) return;
  const int64_t t0 = total * g / parts, t1 = total * (g + 1) / parts;
  const int group = a.q_heads / c.kv_heads;
  const int blocks = (group + AD_ROWS - 1) / AD_ROWS;
  const int kvh = vh / blocks, row0 = (vh - kvh * blocks) * AD_ROWS;
  const int rows = min(AD_ROWS, group - row0);
  const int head0 = kvh * group + row0;
  int seq;
  int64_t before;  // steps before seq
  ad_find<AD_T>(c, s_pre, R, t0, seq, before);

  Q8Ring<HD> ring(c, sc, smem + warp * S::STAGES * S::STAGE_BYTES, s_scale[warp], kvh, seq,
                  (int)(t0 - before), (int)cache_len(c, seq), t1 - t0);
  const float cs = a.scale * 1.4426950408889634f;
  const int r = lane >> 2;
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
    Q8Rows<E, C, HD> w;
    w.start(a, seq, head0, rows);
    w.run(ring, len, j0, j1, cs);
    if (j0 == 0 && j1 == n) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (r + 8 * x >= rows) continue;
        const float f = w.sv / w.l[x];
        char* out = a.out.data + seq * a.out.token_b + (head0 + r + 8 * x) * a.out.head_b;
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const int e = w.element(cc);
          if (e >= c.head_dim) continue;
#pragma unroll
          for (int b = 0; b < S::VB; b += 8) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = w.o[b + i][2 * x + cc] * f;
            *reinterpret_cast<uint4*>(out + 2 * (e + b)) = narrow8<E>(y);
          }
        }
      }
    } else {
      // the part's first piece goes to slot 0, a later one (its last) to slot 1
      const int64_t slot = ((int64_t)(2 * g + (t > t0)) * p.vheads + vh) * AD_ROWS;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int rr = r + 8 * x;
        if (rr >= rows) continue;
        if ((lane & 3) == 0) p.ml[slot + rr] = make_float2(w.mx[x], w.l[x]);
        float* out = p.o + (slot + rr) * p.hd_pad;
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const int e = w.element(cc);
          if (e >= c.head_dim) continue;
#pragma unroll
          for (int b = 0; b < S::VB; b += 4)
            *reinterpret_cast<float4*>(out + e + b) =
                make_float4(w.o[b][2 * x + cc] * w.sv, w.o[b + 1][2 * x + cc] * w.sv,
                            w.o[b + 2][2 * x + cc] * w.sv, w.o[b + 3][2 * x + cc] * w.sv);
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

template <typename E, typename C, int HD>
int launch(const AttnArgs& a, const ScaleView& s, const AdHost& h, void* workspace,
           cudaStream_t stream) {
  static bool set[64] = {};  // per device
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto kern = attention_decode_q8_kernel<E, C, HD>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)Q8Shape<HD>::SMEM));
    if (dev < 64) set[dev] = true;
  }
  const AdPlan p = ad_plan(h, workspace);
  const int st = at_launch(kern, dim3((unsigned)h.grid), Q8Shape<HD>::THREADS, Q8Shape<HD>::SMEM,
                           1, stream, a, s, p);
  if (st != SLS_OK) return st;
  return ad_join<E>(a, p, stream);
}

template <typename E, typename C>
int launch(const AttnArgs& a, const ScaleView& s, const AdHost& h, void* workspace,
           cudaStream_t stream) {
  return a.c.head_dim > 64 ? launch<E, C, 128>(a, s, h, workspace, stream)
                           : launch<E, C, 64>(a, s, h, workspace, stream);
}

int q8_host(const CacheView& c, int q_heads, AdHost* h) {
  return ad_host(c, q_heads, Q8Shape<128>::WARPS, h);
}

}  // namespace

size_t attention_decode_q8_workspace(const CacheView& c, int q_heads) {
  AdHost h;
  if (c.B == 0 || q8_host(c, q_heads, &h) != SLS_OK) return 0;
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
