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

#include "attention_tma.cuh"

namespace sls {

namespace {

__device__ int g_status;  // SLS_ERR_TIMEOUT once a wait gave up

constexpr int AD_KEYS = 32;       // tokens of a step
constexpr int AD_MIN_STEPS = 2;   // a part holds at least so many steps where there are as many
constexpr int AD_ROWS = 16;       // query heads of a tile
constexpr int AD_JOIN_WARPS = 8;
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

// Parts, their groups of warps and the pieces in the workspace.
struct AdPlan {
  int groups;         // most parts
  int vheads;         // key heads times row blocks
  int64_t* prefix;    // B + 1: steps before every sequence
  float2* ml;         // (part, first or last piece, vhead, row): maximum of the scores, sum
  float* o;           // the same, hd_pad elements each
  int hd_pad;
};

SLS_DEV int ad_steps(const CacheView& c, int s) {
  return (int)((cache_len(c, s) + AD_KEYS - 1) / AD_KEYS);
}

SLS_DEV int ad_parts(int64_t total, int groups) {
  const int64_t most = (total + AD_MIN_STEPS - 1) / AD_MIN_STEPS;
  return (int)(most < groups ? most : groups);
}

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
template <typename E>
SLS_DEV void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<E, __nv_bfloat16>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
        "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, "
        "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
  // steps before every chunk of R sequences
  const int R = (c.B + AD_T - 1) / AD_T;
  {
    int64_t mine = 0;
    const int s0 = min(c.B, (int)threadIdx.x * R), s1 = min(c.B, s0 + R);
    for (int s = s0; s < s1; ++s) mine += ad_steps(c, s);
    int64_t pre = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, pre, d);
      if (lane >= d) pre += x;
    }
    if (lane == 31) s_pre[warp] = pre;
    if (lane < S::STAGES) mbar_init(&full_bar[warp][lane], 1);
    mbar_fence_init();
    __syncthreads();
    for (int w = 0; w < warp; ++w) pre += s_pre[w];
    __syncthreads();
    s_pre[threadIdx.x + 1] = pre;
    if (threadIdx.x == 0) s_pre[0] = 0;
    if (blockIdx.x == 0) {
      int64_t at = pre - mine;
      for (int s = s0; s < s1; ++s) {
        p.prefix[s] = at;
        at += ad_steps(c, s);
      }
      if (threadIdx.x == AD_T - 1) p.prefix[c.B] = pre;
    }
    __syncthreads();
  }
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

  // the sequence of step t0
  int seq;
  int64_t before;  // steps before seq
  {
    int lo = 0, hi = AD_T - 1;  // the last chunk that starts at or before t0
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_pre[mid] <= t0) lo = mid;
      else hi = mid - 1;
    }
    seq = lo * R;
    before = s_pre[lo];
    for (;;) {
      const int n = ad_steps(c, seq);
      if (t0 < before + n) break;
      before += n;
      ++seq;
    }
  }

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
  // rows rank, rank + size, ...: the warps of this CTA take the warps of the cluster in
  // turn, in order, then their sums are joined in order
  auto peer = [](const void* p, uint32_t cta) {
    uint32_t x;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(smem_u32(p)), "r"(cta));
    return x;
  };
  auto ld = [](uint32_t x) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(x) : "memory");
    return v;
  };
  auto ld4 = [](uint32_t x) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(x)
                 : "memory");
    return v;
  };
  const int e0 = 4 * lane;
  for (int rr = rank; rr < rows; rr += size) {
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t p = 0; p < size; ++p) {
      // warp `warp` of every CTA's W, CTA by CTA
      const float pm = ld(peer(&s_m[warp][rr], p)), pl = ld(peer(&s_l[warp][rr], p));
      const float4 v =
          e0 < HD ? ld4(peer(out_s + rr * HD + e0, p)) : make_float4(0.f, 0.f, 0.f, 0.f);
      const float mn = fmaxf(m, pm), base = mn == -INFINITY ? 0.f : mn;
      const float f = at_exp2((m - base) * cs), g = at_exp2((pm - base) * cs);
      l = l * f + pl * g;
      o[0] = o[0] * f + v.x * g, o[1] = o[1] * f + v.y * g;
      o[2] = o[2] * f + v.z * g, o[3] = o[3] * f + v.w * g;
      m = mn;
    }
    if (lane == 0) s_join[warp][HD] = m, s_join[warp][HD + 1] = l;
    if (e0 < HD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s_join[warp][e0 + i] = o[i];
    }
    __syncthreads();
    const int e = 2 * threadIdx.x;
    if (e < c.head_dim) {
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < W; ++x) top = fmaxf(top, s_join[x][HD]);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f, y = 0.f, z = 0.f;
#pragma unroll
      for (int x = 0; x < W; ++x) {
        const float f = at_exp2((s_join[x][HD] - base) * cs);
        sum += s_join[x][HD + 1] * f;
        y += s_join[x][e] * f;
        z += s_join[x][e + 1] * f;
      }
      const float inv = n > 0 ? 1.f / sum : 0.f;
      *reinterpret_cast<uint32_t*>(a.out.data + seq * a.out.token_b +
                                   (head0 + rr) * a.out.head_b + 2 * e) =
          Half2<E>::narrow(y * inv, z * inv);
    }
    __syncthreads();
  }
  // no CTA leaves while another reads its shared memory
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Joins the pieces of rows (sequence, query head) in the order of the tokens; zeros for a
// sequence without tokens; nothing to do for one that was not cut.  WARPS warps share a
// row, each a run of its pieces, and join their sums in order at the end; with WARPS = 1 a
// CTA has a row for each of its warps (batches whose sequences have a few pieces each: the
// whole call on 200 sequences of 12 heads 38.5 us with a CTA per row, 35.4 so; 34.9
// since launches overlap).
template <typename E, int WARPS>
__global__ void __launch_bounds__(32 * AD_JOIN_WARPS)
attention_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AdPlan p) {
  __shared__ float s_m[AD_JOIN_WARPS], s_l[AD_JOIN_WARPS];
  __shared__ float s_o[AD_JOIN_WARPS][SLS_MAX_HEAD_DIM];
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  const int warp = WARPS == 1 ? 0 : threadIdx.x >> 5;
  const int64_t row =
      WARPS == 1 ? (int64_t)blockIdx.x * AD_JOIN_WARPS + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= (int64_t)c.B * a.q_heads) return;
  const int seq = (int)(row / a.q_heads), h = (int)(row - (int64_t)seq * a.q_heads);
  const int group = a.q_heads / c.kv_heads, blocks = (group + AD_ROWS - 1) / AD_ROWS;
  const int kvh = h / group, in = h - kvh * group;
  const int vh = kvh * blocks + in / AD_ROWS, rr = in % AD_ROWS;
  char* out = a.out.data + seq * a.out.token_b + h * a.out.head_b;
  const int e0 = 4 * lane;
  at_go();
  at_wait_ahead();
  const int64_t total = p.prefix[c.B], b0 = p.prefix[seq], b1 = p.prefix[seq + 1];
  if (b1 == b0) {
    if (warp == 0 && e0 < c.head_dim)
      *reinterpret_cast<uint2*>(out + 2 * e0) = make_uint2(0u, 0u);
    return;
  }
  const int parts = ad_parts(total, p.groups);
  const float cs = a.scale * 1.4426950408889634f;
  // the part of step t is the last whose start total * g / parts is at most t
  const int g0 = (int)(((b0 + 1) * parts - 1) / total), g1 = (int)((b1 * parts - 1) / total);
  if (g0 == g1) return;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int n = g1 - g0 + 1;
  const int per = (n + WARPS - 1) / WARPS;
  const int x0 = warp * per, x1 = min(n, x0 + per);
#pragma unroll 4
  for (int x = x0; x < x1; ++x) {
    const int g = g0 + x;
    // the sequence's first piece is its part's last unless the part starts with it
    const int late = x == 0 && total * g / parts < b0;
    const int64_t slot = ((int64_t)(2 * g + late) * p.vheads + vh) * AD_ROWS + rr;
    const float2 ml = p.ml[slot];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (e0 < c.head_dim) v = *reinterpret_cast<const float4*>(p.o + slot * p.hd_pad + e0);
    const float mn = fmaxf(m, ml.x), base = mn == -INFINITY ? 0.f : mn;
    const float f = at_exp2((m - base) * cs), w = at_exp2((ml.x - base) * cs);
    l = l * f + ml.y * w;
    o[0] = o[0] * f + v.x * w, o[1] = o[1] * f + v.y * w;
    o[2] = o[2] * f + v.z * w, o[3] = o[3] * f + v.w * w;
    m = mn;
  }
  if constexpr (WARPS == 1) {
    const float inv = 1.f / l;
    if (e0 < c.head_dim)
      *reinterpret_cast<uint2*>(out + 2 * e0) =
          make_uint2(Half2<E>::narrow(o[0] * inv, o[1] * inv),
                     Half2<E>::narrow(o[2] * inv, o[3] * inv));
    return;
  }
  if (lane == 0) s_m[warp] = m, s_l[warp] = l;
  *reinterpret_cast<float4*>(&s_o[warp][e0]) = make_float4(o[0], o[1], o[2], o[3]);
  __syncthreads();
  const int e = threadIdx.x;
  if (2 * e < c.head_dim) {
    float top = -INFINITY;
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_m[w]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f, x = 0.f, y = 0.f;
    for (int w = 0; w < WARPS; ++w) {
      if (w * per >= n) break;
      const float f = at_exp2((s_m[w] - base) * cs);
      sum += s_l[w] * f;
      x += s_o[w][2 * e] * f;
      y += s_o[w][2 * e + 1] * f;
    }
    const float inv = 1.f / sum;
    *reinterpret_cast<uint32_t*>(out + 4 * e) = Half2<E>::narrow(x * inv, y * inv);
  }
}

// Parts, and the workspace's layout.
struct AdHost {
  int cluster;  // CTAs of a cluster; 0: parts and pieces
  int groups, vheads, grid, hd_pad;
  size_t prefix_b, ml_b, o_b;
};

int ad_host(const CacheView& c, int q_heads, AdHost* h) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int warps = c.head_dim > 64 ? AdShape<128>::WARPS : AdShape<64>::WARPS;
  const int group = q_heads / c.kv_heads, blocks = (group + AD_ROWS - 1) / AD_ROWS;
  h->vheads = c.kv_heads * blocks;
  // A cluster for each (sequence, key head) where they and their CTAs fit the GPU at once
  // (a CTA each: twice) and no warp gets more than 16 steps; up to 16 query heads a key
  // head, so that a key is read once.  Device time of parts and pieces / clusters, 28 + 4
  // heads, before launches overlapped: 1 x 2061 tokens 9.8 / 6.9 us, 32 x 500 13.4 / 8.8
  // (a CTA each, as the next), 64 x 1000 25.4 / 23.6; 100 x 300, more than twice, 16.6 / 20.4.
  h->cluster = 0;
  const int64_t units = (int64_t)c.B * h->vheads, room = (int64_t)c.max_pages << c.page_shift;
  if (blocks == 1)
    for (int n = 8; n >= 1 && h->cluster == 0; n /= 2)
      if (units * n <= (n == 1 ? 2 : 1) * sms && room <= (int64_t)16 * AD_KEYS * n * warps) h->cluster = n;
  h->groups = std::max(1, sms * warps / h->vheads);
  // no more parts than the page tables can hold steps for
  const int64_t most = (int64_t)c.B * (((int64_t)c.max_pages << c.page_shift) / AD_KEYS + 1);
  h->groups = (int)std::min<int64_t>(h->groups, (most + AD_MIN_STEPS - 1) / AD_MIN_STEPS);
  h->grid = (h->groups * h->vheads + warps - 1) / warps;
  h->hd_pad = c.head_dim;
  h->prefix_b = sls_align256(((size_t)c.B + 1) * 8);
  const size_t rows = (size_t)h->groups * 2 * h->vheads * AD_ROWS;
  h->ml_b = sls_align256(rows * 8);
  h->o_b = sls_align256(rows * h->hd_pad * 4);
  return SLS_OK;
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
  // a sequence has 1 + groups / B pieces on average
  const bool few = p.groups <= 2 * (int64_t)a.c.B;
  const int64_t rows = (int64_t)a.c.B * a.q_heads;
  return at_launch(few ? attention_join_kernel<E, 1> : attention_join_kernel<E, AD_JOIN_WARPS>,
                   dim3((unsigned)(few ? (rows + AD_JOIN_WARPS - 1) / AD_JOIN_WARPS : rows)),
                   32 * AD_JOIN_WARPS, 0, 1, stream, a, p);
}

}  // namespace

size_t attention_decode_workspace(const CacheView& c, int q_heads) {
  AdHost h;
  if (c.B == 0 || ad_host(c, q_heads, &h) != SLS_OK || h.cluster > 0) return 0;
  return h.prefix_b + h.ml_b + h.o_b;
}

int launch_attention_decode(const AttnArgs& a, int dtype, void* workspace, cudaStream_t stream) {
  const CacheView& c = a.c;
  if (c.B == 0) return SLS_OK;
  AdHost h;
  int st = ad_host(c, a.q_heads, &h);
  if (st != SLS_OK) return st;
  if ((int64_t)c.B * a.q_heads > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  AdPlan p;
  p.groups = h.groups;
  p.vheads = h.vheads;
  p.hd_pad = h.hd_pad;
  p.prefix = (int64_t*)workspace;
  p.ml = (float2*)((char*)workspace + h.prefix_b);
  p.o = (float*)((char*)workspace + h.prefix_b + h.ml_b);
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
