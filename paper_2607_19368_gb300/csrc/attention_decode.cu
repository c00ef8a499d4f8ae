// One new token per sequence over the paged cache: o = softmax(scale q K^T) V for
// every query head, K and V of the sequence's length read once.
//
// Bound by HBM bandwidth: 4 hd bytes a cached token and key head against
// 4 hd G operations (G query heads per key head).  A warp owns a (sequence, key
// head) at a time: the G rows of its group fill part of a 16-row mma.sync tile
// (the tcgen05 tiles of 64 and more rows would be filled to a few percent, and the
// products take 10% of the time that the bytes take), scores, weights and the
// 16 x hd outputs stay in its registers, and keys and values come through its own
// ring of 128-byte-swizzled shared-memory stages (32 tokens each) by TMA, so warps
// never wait for one another.  The warps of adjacent key heads walk the same
// tokens at the same time, which makes their reads adjacent in memory.
//
// All sequences' steps of 32 tokens form one list, cut into equal parts, one for
// each group of kv_heads warps: lengths may be as uneven as they like.  A part that
// holds all of a sequence writes its result; pieces of a sequence leave their
// unnormalised sums, maxima and weight sums in the workspace, and a second small
// launch joins them in the order of the tokens.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "attention_decode.cuh"

namespace sls {

namespace {

__device__ int g_status;  // SLS_ERR_TIMEOUT once a wait gave up

// log2 of a factor of all weights, which the division by their sum takes out again: float16
// weights use the range above 1 too, so that many small ones next to a large one (2^-25 and
// less of it, which would round to 0) reach the output as they reach the sum
template <typename E>
constexpr float AD_SHIFT = std::is_same<E, __nv_bfloat16>::value ? 0.f : 15.f;

template <int HD>
struct AdShape {
  static constexpr int HALVES = HD / 64;
  static constexpr int HALF_BYTES = AD_KEYS * 128;
  static constexpr int MAT_BYTES = HALVES * HALF_BYTES;  // K or V of a step
  static constexpr int STAGE_BYTES = 2 * MAT_BYTES;
  // narrow heads have half the bytes a step and nearly the same instructions: twice the
  // warps
  static constexpr int WARPS = HD == 128 ? 4 : 8;
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int STAGES = 3;
  static constexpr size_t SMEM = (size_t)WARPS * STAGES * STAGE_BYTES + 1024;
};

SLS_DEV void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
SLS_DEV void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// A warp's ring: its next steps are copied ahead, from sequence to sequence.
template <int HD>
struct AdRing {
  using S = AdShape<HD>;
  const CacheView& c;
  const CUtensorMap* tmK;
  const CUtensorMap* tmV;
  unsigned char* mem;
  uint64_t* bars;
  int kvh;
  uint32_t lead;
  int is, ij, ilen;  // the step to issue next: its sequence, its number there, the length
  int64_t left;      // steps still to issue
  int batch0, page;  // lane l: the page of tokens 16 l of the batch of 16 steps from batch0 on
  unsigned issued, used;

  SLS_DEV AdRing(const CacheView& cache, const CUtensorMap* k, const CUtensorMap* v,
                 unsigned char* ring, uint64_t* b, int head, int seq, int step, int len, int64_t n)
      : c(cache), tmK(k), tmV(v), mem(ring), bars(b), kvh(head), lead(at_elect()), is(seq),
        ij(step), ilen(len), left(n), batch0(-1), page(-1), issued(0), used(0) {
#pragma unroll 1
    for (int i = 0; i < S::STAGES; ++i) issue();
  }

  SLS_DEV void issue() {
    if (left == 0) return;
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
    if (lead) mbar_expect_tx(&bars[st], 2 * S::HALVES * copies * box * 128);
    __syncwarp();
#pragma unroll 1
    for (int cp = 0; cp < copies; ++cp) {
      const int pg = __shfl_sync(0xffffffffu, page, 2 * (ij - batch0) + cp);
      const uint32_t dst = smem_u32(mem) + st * S::STAGE_BYTES + cp * box * 128;
#pragma unroll
      for (int h = 0; h < S::HALVES; ++h) {
        at_tma4(lead, dst + h * S::HALF_BYTES, tmK, 64 * h, slot0, kvh, pg, &bars[st]);
        at_tma4(lead, dst + S::MAT_BYTES + h * S::HALF_BYTES, tmV, 64 * h, slot0, kvh, pg,
                &bars[st]);
      }
    }
    ++ij;
    ++issued;
    --left;
  }

  // Waits for the next step; false when the time is up, after the other copies in
  // flight have landed or run out of time too.
  SLS_DEV bool wait() {
    if (__all_sync(0xffffffffu, mbar_wait(&bars[used % S::STAGES], (used / S::STAGES) & 1)))
      return true;
    if ((threadIdx.x & 31) == 0) atomicExch(&g_status, SLS_ERR_TIMEOUT);
    for (unsigned x = used + 1; x < issued; ++x)
      mbar_wait(&bars[x % S::STAGES], (x / S::STAGES) & 1);
    return false;
  }
};

// The rows of a piece: queries as A fragments, unnormalised outputs, the maximum in use
// and this lane's part of the sum of weights, for rows lane / 4 and lane / 4 + 8.
template <typename E, int HD>
struct AdRows {
  using S = AdShape<HD>;
  static constexpr int KS = HD / 16;  // 16-element slices of a head
  static constexpr int NB = HD / 8;   // 8-element blocks of a head
  uint32_t q[KS][4];
  float o[NB][4];
  float mx[2], l[2];

  SLS_DEV void start(const AttnArgs& a, int seq, int head0, int rows) {
    const int lane = threadIdx.x & 31, r = lane >> 2, cq = 2 * (lane & 3);
    const char* qp = a.q.data + seq * a.q.token_b + head0 * a.q.head_b;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rr = r + 8 * (i & 1), e = 16 * k + cq + 8 * (i >> 1);
        q[k][i] = (rr < rows && e < a.c.head_dim)
                      ? *reinterpret_cast<const uint32_t*>(qp + rr * a.q.head_b + 2 * e)
                      : 0u;
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b][0] = o[b][1] = o[b][2] = o[b][3] = 0.f;
    mx[0] = mx[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }

  // steps [j0, j1) of a sequence of `len` tokens; cs: scale log2(e)
  SLS_DEV bool run(AdRing<HD>& ring, int len, int j0, int j1, float cs) {
    const int lane = threadIdx.x & 31, cq = 2 * (lane & 3);
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
      if (!ring.wait()) return false;
      unsigned char* stage = ring.mem + (ring.used % S::STAGES) * S::STAGE_BYTES;
      const uint32_t kb = smem_u32(stage), vb = kb + S::MAT_BYTES;
      const int lim = len - j * AD_KEYS;
      if (lim < AD_KEYS) {
        // values past the end: whatever their slots hold, zero here
        unsigned char* v = stage + S::MAT_BYTES;
        for (int x = lim * 8 + lane; x < AD_KEYS * 8; x += 32)
#pragma unroll
          for (int h = 0; h < S::HALVES; ++h)
            reinterpret_cast<uint4*>(v + h * S::HALF_BYTES)[x] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      float s[4][4];
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
        const int row = nb * 8 + (lane & 7);
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
          const int ch = 4 * i + (lane >> 3);
          uint32_t b[4];
          ldsm4(kb + (ch >> 3) * S::HALF_BYTES + row * 128 + (((ch & 7) ^ (row & 7)) << 4), b);
          mma16816<E>(s[nb], q[2 * i], b[0], b[1]);
          mma16816<E>(s[nb], q[2 * i + 1], b[2], b[3]);
        }
      }
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
      if (__any_sync(0xffffffffu, top[0] > mx[0] || top[1] > mx[1])) {
        float f[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          f[x] = top[x] > mx[x] ? at_exp2((mx[x] - top[x]) * cs) : 1.f;
          mx[x] = top[x];
          l[x] *= f[x];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          o[b][0] *= f[0], o[b][1] *= f[0];
          o[b][2] *= f[1], o[b][3] *= f[1];
        }
      }
      // the distance from the maximum first, which is exact where it matters: scale times
      // maximum would round by more than the weights' range where scores are large
      const float base[2] = {mx[0] == -INFINITY ? 0.f : mx[0], mx[1] == -INFINITY ? 0.f : mx[1]};
      uint32_t w[2][4];
      float sum[2] = {0.f, 0.f};  // of the step: added to l one by one, small weights next to a
                                  // large one would be below half of its last place
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[i] = at_exp2(__fmaf_rn(s[nb][i] - base[i >> 1], cs, AD_SHIFT<E>));
          sum[i >> 1] += e[i];
        }
        w[nb >> 1][2 * (nb & 1)] = Half2<E>::narrow(e[0], e[1]);
        w[nb >> 1][2 * (nb & 1) + 1] = Half2<E>::narrow(e[2], e[3]);
      }
      l[0] += sum[0], l[1] += sum[1];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int row = ks * 16 + (lane & 15);
#pragma unroll
        for (int b = 0; b < NB; b += 2) {
          const int ch = b + (lane >> 4);
          uint32_t v[4];
          ldsm4t(vb + (ch >> 3) * S::HALF_BYTES + row * 128 + (((ch & 7) ^ (row & 7)) << 4), v);
          mma16816<E>(o[b], w[ks], v[0], v[1]);
          mma16816<E>(o[b + 1], w[ks], v[2], v[3]);
        }
      }
      __syncwarp();
      ++ring.used;
      ring.issue();
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
    }
    return true;
  }
};

template <typename E, int HD>
__global__ void __launch_bounds__(AdShape<HD>::THREADS, 1)
attention_decode_kernel(const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV,
                        const __grid_constant__ AttnArgs a, const __grid_constant__ AdPlan p) {
  using S = AdShape<HD>;
  constexpr int AD_T = S::THREADS;
  constexpr int NB = HD / 8;  // 8-element blocks of a head
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t full_bar[S::WARPS][S::STAGES];
  __shared__ int64_t s_pre[AD_T + 1];
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
  AdRing<HD> ring(c, &tmK, &tmV, smem + warp * S::STAGES * S::STAGE_BYTES, full_bar[warp], kvh,
                  seq, (int)(t0 - before), (int)cache_len(c, seq), t1 - t0);

  const float cs = a.scale * 1.4426950408889634f;
  const int r = lane >> 2, cq = 2 * (lane & 3);
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
    AdRows<E, HD> w;
    w.start(a, seq, head0, rows);
    if (!w.run(ring, len, j0, j1, cs)) return;
    const auto& o = w.o;
    const float(&mx)[2] = w.mx, (&l)[2] = w.l;
    if (j0 == 0 && j1 == n) {
      const float inv[2] = {1.f / l[0], 1.f / l[1]};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (r + 8 * x >= rows) continue;
        char* out = a.out.data + seq * a.out.token_b + (head0 + r + 8 * x) * a.out.head_b;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          if (8 * b + cq < c.head_dim)
            *reinterpret_cast<uint32_t*>(out + 2 * (8 * b + cq)) =
                Half2<E>::narrow(o[b][2 * x] * inv[x], o[b][2 * x + 1] * inv[x]);
      }
    } else {
      // the part's first piece goes to slot 0, a later one (its last) to slot 1
      const int64_t slot = ((int64_t)(2 * g + (t > t0)) * p.vheads + vh) * AD_ROWS;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int rr = r + 8 * x;
        if (rr >= rows) continue;
        if (cq == 0)
          p.ml[slot + rr] = make_float2(mx[x], l[x]);
        float* out = p.o + (slot + rr) * p.hd_pad;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          if (8 * b + cq < p.hd_pad)
            *reinterpret_cast<float2*>(out + 8 * b + cq) =
                make_float2(o[b][2 * x], o[b][2 * x + 1]);
      }
    }
    t = before + j1;
    if (j1 == n) {
      before += n;
      ++seq;
    }
  }
}

// Few rows: a cluster of CTAs owns a (sequence, key head, block of rows), its warps take
// equal pieces of the sequence, leave maximum, sum and unnormalised output in shared
// memory, and the CTAs join the rows among themselves (row r by CTA r mod size) reading
// one another's shared memory: one launch, no workspace.
template <typename E, int HD>
__global__ void __launch_bounds__(AdShape<HD>::THREADS, 1)
attention_decode_cluster_kernel(const __grid_constant__ CUtensorMap tmK,
                                const __grid_constant__ CUtensorMap tmV,
                                const __grid_constant__ AttnArgs a, int vheads) {
  using S = AdShape<HD>;
  constexpr int NB = HD / 8;
  constexpr int W = S::WARPS;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t full_bar[W][S::STAGES];
  __shared__ float s_m[W][AD_ROWS], s_l[W][AD_ROWS];
  __shared__ float s_join[W][HD + 2];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int unit = blockIdx.x / size;
  const int seq = unit / vheads, vh = unit - seq * vheads;
  const int group = a.q_heads / c.kv_heads;
  const int blocks = (group + AD_ROWS - 1) / AD_ROWS;
  const int kvh = vh / blocks, row0 = (vh - kvh * blocks) * AD_ROWS;
  const int rows = min(AD_ROWS, group - row0);
  const int head0 = kvh * group + row0;
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
  AdRing<HD> ring(c, &tmK, &tmV, mine, full_bar[warp], kvh, seq, j0, len, j1 - j0);
  AdRows<E, HD> w;
  w.start(a, seq, head0, rows);
  const float cs = a.scale * 1.4426950408889634f;
  const bool ok = w.run(ring, len, j0, j1, cs);
  // the outputs go where the warp's ring was: 16 rows of HD floats
  static_assert(S::STAGES * S::STAGE_BYTES >= AD_ROWS * HD * 4, "a ring holds a piece");
  const int r = lane >> 2, cq = 2 * (lane & 3);
  float* out_s = reinterpret_cast<float*>(mine);
  __syncwarp();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int rr = r + 8 * x;
    if (cq == 0) {
      s_m[warp][rr] = w.mx[x];
      s_l[warp][rr] = ok ? w.l[x] : 0.f;
    }
    if (rr < rows) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<float2*>(out_s + rr * HD + 8 * b + cq) =
            make_float2(w.o[b][2 * x], w.o[b][2 * x + 1]);
    }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  ad_cluster_join<E, HD, W>(a, seq, head0, rows, n, rank, size, cs, s_m[0], s_l[0], AD_ROWS, out_s,
                            s_join);
  // no CTA leaves while another reads its shared memory
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

int ad_warps(const CacheView& c) {
  return c.head_dim > 64 ? AdShape<128>::WARPS : AdShape<64>::WARPS;
}

template <typename E, int HD>
int launch_cluster(const AttnArgs& a, const AdHost& h, const CUtensorMap& k, const CUtensorMap& v,
                   cudaStream_t stream) {
  static bool set[64] = {};  // per device
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto kern = attention_decode_cluster_kernel<E, HD>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)AdShape<HD>::SMEM));
    if (dev < 64) set[dev] = true;
  }
  return at_launch(kern, dim3((unsigned)(a.c.B * h.vheads * h.cluster)), AdShape<HD>::THREADS,
                   AdShape<HD>::SMEM, h.cluster, stream, k, v, a, h.vheads);
}

template <typename E, int HD>
int launch(const AttnArgs& a, const AdPlan& p, int grid, const CUtensorMap& k,
           const CUtensorMap& v, cudaStream_t stream) {
  static bool set[64] = {};  // per device
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto kern = attention_decode_kernel<E, HD>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)AdShape<HD>::SMEM));
    if (dev < 64) set[dev] = true;
  }
  const int st = at_launch(kern, dim3((unsigned)grid), AdShape<HD>::THREADS, AdShape<HD>::SMEM, 1,
                           stream, k, v, a, p);
  if (st != SLS_OK) return st;
  return ad_join<E>(a, p, stream);
}

}  // namespace

size_t attention_decode_workspace(const CacheView& c, int q_heads) {
  AdHost h;
  if (c.B == 0 || ad_host(c, q_heads, ad_warps(c), &h) != SLS_OK || h.cluster > 0) return 0;
  return h.prefix_b + h.ml_b + h.o_b;
}

int launch_attention_decode(const AttnArgs& a, int dtype, void* workspace, cudaStream_t stream) {
  const CacheView& c = a.c;
  if (c.B == 0) return SLS_OK;
  AdHost h;
  int st = ad_host(c, a.q_heads, ad_warps(c), &h);
  if (st != SLS_OK) return st;
  if ((int64_t)c.B * a.q_heads > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  const AdPlan p = ad_plan(h, workspace);
  CUtensorMap k, v;
  if (!at_cache_map(&k, dtype, c, c.k, std::min(AD_KEYS, 1 << c.page_shift)) ||
      !at_cache_map(&v, dtype, c, c.v, std::min(AD_KEYS, 1 << c.page_shift)))
    return SLS_ERR_UNSUPPORTED;
  const bool wide = c.head_dim > 64;
  if (h.cluster > 0) {
    if (dtype == SLS_BF16)
      return wide ? launch_cluster<__nv_bfloat16, 128>(a, h, k, v, stream)
                  : launch_cluster<__nv_bfloat16, 64>(a, h, k, v, stream);
    return wide ? launch_cluster<__half, 128>(a, h, k, v, stream)
                : launch_cluster<__half, 64>(a, h, k, v, stream);
  }
  if (dtype == SLS_BF16)
    return wide ? launch<__nv_bfloat16, 128>(a, p, h.grid, k, v, stream)
                : launch<__nv_bfloat16, 64>(a, p, h.grid, k, v, stream);
  return wide ? launch<__half, 128>(a, p, h.grid, k, v, stream)
              : launch<__half, 64>(a, p, h.grid, k, v, stream);
}

int decode_status_word(int** word) {
  void* p = nullptr;
  SLS_CUDA_TRY(cudaGetSymbolAddress(&p, g_status));
  *word = (int*)p;
  return SLS_OK;
}

}  // namespace sls
