// What the decode kernels share, over 16 bits and over codes: parts of the list of all
// sequences' steps, the workspace's pieces and their joining.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attention_tma.cuh"

namespace sls {

constexpr int AD_KEYS = 32;       // tokens of a step
constexpr int AD_MIN_STEPS = 2;   // a part holds at least so many steps where there are as many
constexpr int AD_ROWS = 16;       // query heads of a tile
constexpr int AD_JOIN_WARPS = 8;

// Parts, their groups of warps and the pieces in the workspace.
struct AdPlan {
  int groups;         // most parts
  int vheads;         // key heads times row blocks
  int64_t* prefix;    // B + 1: steps before every sequence
  float2* ml;         // (part, first or last piece, vhead, row): maximum of the scores, sum
  float* o;           // the same, hd_pad elements each
  int hd_pad;
};

// Steps of KEYS tokens of sequence s.
template <int KEYS = AD_KEYS>
SLS_DEV int ad_steps(const CacheView& c, int s) {
  return (int)((cache_len(c, s) + KEYS - 1) / KEYS);
}

SLS_DEV int ad_parts(int64_t total, int groups) {
  const int64_t most = (total + AD_MIN_STEPS - 1) / AD_MIN_STEPS;
  return (int)(most < groups ? most : groups);
}

// Steps before every chunk of R sequences, for the CTA's T threads: s_pre[i] those before
// chunk i, s_pre[T] all; steps(s): those of sequence s.  CTA 0 writes those before every sequence
// to `prefix`, if given.  Returns R.
template <int T, typename F>
SLS_DEV int ad_prefix(const CacheView& c, int64_t* s_pre, int64_t* prefix, const F& steps) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = (c.B + T - 1) / T;
  int64_t mine = 0;
  const int s0 = min(c.B, (int)threadIdx.x * R), s1 = min(c.B, s0 + R);
  for (int s = s0; s < s1; ++s) mine += steps(s);
  int64_t pre = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, pre, d);
    if (lane >= d) pre += x;
  }
  if (lane == 31) s_pre[warp] = pre;
  __syncthreads();
  for (int w = 0; w < warp; ++w) pre += s_pre[w];
  __syncthreads();
  s_pre[threadIdx.x + 1] = pre;
  if (threadIdx.x == 0) s_pre[0] = 0;
  if (prefix && blockIdx.x == 0) {
    int64_t at = pre - mine;
    for (int s = s0; s < s1; ++s) {
      prefix[s] = at;
      at += steps(s);
    }
    if (threadIdx.x == T - 1) prefix[c.B] = pre;
  }
  __syncthreads();
  return R;
}

// x / y, neither negative, in 32 bits where that is enough: a division in 64 takes some hundred
// instructions, which a small call fetches for the first time as a rule.
SLS_DEV int64_t ad_div(int64_t x, int64_t y) {
  return (uint64_t)(x | y) >> 32 ? x / y : (int64_t)((unsigned)x / (unsigned)y);
}

// The sequence of step t0 (below the total), and the steps before it.
template <int T, typename F>
SLS_DEV void ad_find(const int64_t* s_pre, int R, int64_t t0, const F& steps, int& seq,
                     int64_t& before) {
  int lo = 0, hi = T - 1;  // the last chunk that starts at or before t0
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s_pre[mid] <= t0) lo = mid;
    else hi = mid - 1;
  }
  seq = lo * R;
  before = s_pre[lo];
  for (;;) {
    const int64_t n = steps(seq);
    if (t0 < before + n) break;
    before += n;
    ++seq;
  }
}

// Token of row j of an operand of sixteen, where a lane reads its fragments by whole 16 bytes:
// tokens 2 c and 2 c + 1 are 2 c and (2 c ^ 4) + 1 of the cache, so that neither reads of keys (four
// chunks of two rows) nor of values (two of four) meet a bank twice.
SLS_DEV int ad_token(int j) { return j ^ (j & 1) << 2; }

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

// The rows of a cluster whose W warps a CTA left maxima and sums (warp by warp, `pitch` rows each) and
// unnormalised outputs (HD floats a row, `out_s` for this warp) in shared memory; n: the steps of
// the sequence.
template <typename E, int HD, int W>
SLS_DEV void ad_cluster_join(const AttnArgs& a, int seq, int head0, int rows, int n, uint32_t rank,
                             uint32_t size, float cs, const float* s_m, const float* s_l, int pitch,
                             const float* out_s, float (*s_join)[HD + 2]) {
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
      const float pm = ld(peer(s_m + warp * pitch + rr, p)), pl = ld(peer(s_l + warp * pitch + rr, p));
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
  const int seq = (int)ad_div(row, a.q_heads), h = (int)(row - (int64_t)seq * a.q_heads);
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
  const int g0 = (int)ad_div((b0 + 1) * parts - 1, total), g1 = (int)ad_div(b1 * parts - 1, total);
  if (g0 == g1) return;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int n = g1 - g0 + 1;
  const int per = (n + WARPS - 1) / WARPS;
  const int x0 = warp * per, x1 = min(n, x0 + per);
#pragma unroll 4
  for (int x = x0; x < x1; ++x) {
    const int g = g0 + x;
    // the sequence's first piece is its part's last unless the part starts with it
    const int late = x == 0 && ad_div(total * g, parts) < b0;
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

// warps: of a CTA (one CTA per SM)
inline int ad_host(const CacheView& c, int q_heads, int warps, AdHost* h) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
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

inline AdPlan ad_plan(const AdHost& h, void* workspace) {
  AdPlan p;
  p.groups = h.groups;
  p.vheads = h.vheads;
  p.hd_pad = h.hd_pad;
  p.prefix = (int64_t*)workspace;
  p.ml = (float2*)((char*)workspace + h.prefix_b);
  p.o = (float*)((char*)workspace + h.prefix_b + h.ml_b);
  return p;
}

template <typename E>
int ad_join(const AttnArgs& a, const AdPlan& p, cudaStream_t stream) {
  // a sequence has 1 + groups / B pieces on average
  const bool few = p.groups <= 2 * (int64_t)a.c.B;
  const int64_t rows = (int64_t)a.c.B * a.q_heads;
  return at_launch(few ? attention_join_kernel<E, 1> : attention_join_kernel<E, AD_JOIN_WARPS>,
                   dim3((unsigned)(few ? (rows + AD_JOIN_WARPS - 1) / AD_JOIN_WARPS : rows)),
                   32 * AD_JOIN_WARPS, 0, 1, stream, a, p);
}

}  // namespace sls
