// Eviction: of every (sequence, key head) the first and last tokens and the heaviest others
// stay, in order, and move to the front of the sequence's pages.
//
// Two launches.  The first selects: the weight that the last of the kept others has is found
// digit by digit (counts of 2048, 2048 and 1024 digits of the weights as ordered integers), then
// the tokens are gone through once in order, which gives every kept one its place; weights move
// here.  The second moves keys and values.  A place is never behind its source, so a cluster of
// CTAs takes the places in waves, in order: what a wave reads lies at or behind its first place,
// what earlier waves wrote lies in front of it, and the one barrier between a wave's reads and its
// writes is all that moving in place needs.  Bound by the bytes of weights and moved rows.
#include <algorithm>

#include "cache8.cuh"

namespace sls {

namespace {

constexpr int EV_T = 1024;    // selection
constexpr int EV_BINS = 2048;
constexpr int EV_MOVE_T = 256;
constexpr int EV_ROWS = 128;  // rows of a CTA's wave: whole blocks of codes
constexpr int EV_CLUSTER = 8;

// Weights as integers in their order: NaN first, the two zeros equal.
SLS_DEV uint32_t ev_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

struct EvSeq {
  const EvictArgs& a;
  int seq, h;
  // a weight's address, or NULL outside the cache
  SLS_DEV float* weight(int64_t x) const {
    const int64_t page = a.c.table[seq * a.c.table_ld + (x >> a.c.page_shift)];
    if (page < 0 || page >= a.c.num_pages) return nullptr;
    return a.w.data + page * a.w.page + h * a.w.head + (x & ((1 << a.c.page_shift) - 1));
  }
};

__global__ void __launch_bounds__(EV_T)
cache_evict_select_kernel(const __grid_constant__ EvictArgs a, int32_t* lens_before) {
  __shared__ unsigned s_bins[EV_BINS];
  __shared__ unsigned s_warp[EV_T / 32][2];
  __shared__ unsigned s_digit, s_above;
  const CacheView& c = a.c;
  const int seq = blockIdx.x / c.kv_heads, h = blockIdx.x - seq * c.kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  at_go();
  at_wait_ahead();
  const int len = (int)cache_len(c, seq);
  if (h == 0 && threadIdx.x == 0) lens_before[seq] = len;
  int32_t* kept = a.kept + ((int64_t)seq * c.kv_heads + h) * a.keep;
  if (len <= a.keep) {
    for (int i = threadIdx.x; i < a.keep; i += EV_T) kept[i] = i < len ? i : -1;
    return;
  }
  const EvSeq e{a, seq, h};
  const int lo = a.first, hi = len - a.last;
  unsigned need = (unsigned)(a.keep - a.first - a.last);
  // ---- the need-th largest of [lo, hi): its digits from the top, and how many equal it are kept
  uint32_t top = 0, mask = 0;
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    for (int i = threadIdx.x; i < EV_BINS; i += EV_T) s_bins[i] = 0;
    __syncthreads();
    for (int x = lo + threadIdx.x; x < hi; x += EV_T) {
      const float* w = e.weight(x);
      const uint32_t k = ev_key(w ? *w : 0.f);
      if ((k & mask) == top) atomicAdd(&s_bins[(k >> shift) & digits], 1u);
    }
    __syncthreads();
    // the digit at which the count from the top reaches `need`
    const int b = EV_BINS - 1 - 2 * threadIdx.x;  // this thread's larger digit
    const unsigned n0 = s_bins[b], n1 = s_bins[b - 1];
    unsigned sum = n0 + n1;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned y = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += y;
    }
    if (lane == 31) s_warp[warp][0] = sum;
    __syncthreads();
    unsigned above = sum - n0 - n1;
    for (int w = 0; w < warp; ++w) above += s_warp[w][0];
    if (above < need && need <= above + n0) s_digit = b, s_above = above;
    else if (above + n0 < need && need <= above + n0 + n1) s_digit = b - 1, s_above = above + n0;
    __syncthreads();
    top |= s_digit << shift;
    mask |= digits << shift;
    need -= s_above;
    __syncthreads();
  }
  // ---- in order: larger ones and the first `need` equal ones stay
  unsigned base_more = 0, base_same = 0;
  for (int x0 = 0; x0 < len; x0 += EV_T) {
    const int x = x0 + threadIdx.x;
    float w = 0.f;
    bool more = false, same = false;
    if (x < len) {
      const float* p = e.weight(x);
      w = p ? *p : 0.f;
      const uint32_t k = ev_key(w);
      more = x < lo || x >= hi || (mask != 0 && k > top);
      same = !more && mask != 0 && k == top;
    }
    const unsigned bm = __ballot_sync(0xffffffffu, more), bs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) s_warp[warp][0] = __popc(bm), s_warp[warp][1] = __popc(bs);
    __syncthreads();  // the tile's weights are read, too
    const unsigned low = (1u << lane) - 1;
    unsigned m = base_more + __popc(bm & low), s = base_same + __popc(bs & low);
    unsigned all_m = 0, all_s = 0;
    for (int v = 0; v < EV_T / 32; ++v) {
      if (v < warp) m += s_warp[v][0], s += s_warp[v][1];
      all_m += s_warp[v][0], all_s += s_warp[v][1];
    }
    base_more += all_m, base_same += all_s;
    if (more || (same && s < need)) {
      const unsigned to = m + min(s, need);
      kept[to] = x;
      if (to != (unsigned)x)
        if (float* p = e.weight(to)) *p = w;
    }
    __syncthreads();
  }
  for (int x = a.keep + threadIdx.x; x < len; x += EV_T)
    if (float* p = e.weight(x)) *p = 0.f;
}

SLS_DEV void ev_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// C: I8 or E4M3, or void for 16-bit elements
template <typename C>
__global__ void __launch_bounds__(EV_MOVE_T)
cache_evict_move_kernel(const __grid_constant__ EvictArgs a, const int32_t* lens_before) {
  constexpr bool CODES = !std::is_void<C>::value;
  // vectors of 16 bytes of a thread: 128 rows of up to 256 (128) bytes
  constexpr int V = EV_ROWS * SLS_MAX_HEAD_DIM * (CODES ? 1 : 2) / 16 / EV_MOVE_T;
  __shared__ float s_was[EV_ROWS];
  const CacheView& c = a.c;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int unit = blockIdx.x / size;
  const int heads = 2 * c.kv_heads;
  const int seq = unit / heads, hk = unit - seq * heads;
  const bool keys = hk < c.kv_heads;
  const int h = keys ? hk : hk - c.kv_heads;
  at_go();
  at_wait_ahead();
  const int len = lens_before[seq];
  if (len <= a.keep) return;  // the whole cluster
  if (hk == 0 && rank == 0 && threadIdx.x == 0) a.lens[seq] = a.keep;
  const int32_t* kept = a.kept + ((int64_t)seq * c.kv_heads + h) * a.keep;
  const int32_t* table = c.table + seq * c.table_ld;
  char* data = (keys ? c.k : c.v) + h * c.head_b;
  float* scale = CODES ? (keys ? a.s.k : a.s.v) + h * a.s.head : nullptr;
  const int vecs = c.head_dim * (CODES ? 1 : 2) / 16;
  const int slots = (1 << c.page_shift) - 1;
  auto page_of = [&](int x) {
    const int64_t p = table[x >> c.page_shift];
    return p >= 0 && p < c.num_pages ? p : (int64_t)-1;
  };
  for (int w0 = 0; w0 < a.keep; w0 += EV_ROWS * (int)size) {
    const int j0 = w0 + (int)rank * EV_ROWS;
    const int n = min(EV_ROWS, a.keep - j0);
    uint4 x[V];
    if constexpr (CODES) {
      if (threadIdx.x < EV_ROWS) {
        float f = 0.f;
        if ((int)threadIdx.x < n) {
          const int src = kept[j0 + threadIdx.x];
          const int64_t p = page_of(src);
          if (p >= 0) f = scale[p * a.s.page + ((src & slots) >> a.s.shift) * a.s.block];
        }
        s_was[threadIdx.x] = f;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = i * EV_MOVE_T + threadIdx.x, row = at / vecs;
      x[i] = make_uint4(0, 0, 0, 0);
      if (row >= n) continue;
      const int src = kept[j0 + row];
      const int64_t p = page_of(src);
      if (p >= 0)
        x[i] = *reinterpret_cast<const uint4*>(data + p * c.page_b + (src & slots) * c.slot_b +
                                               16 * (at - row * vecs));
    }
    ev_cluster_sync();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = i * EV_MOVE_T + threadIdx.x, row = at / vecs;
      if (row >= n) continue;
      const int64_t p = page_of(j0 + row);
      if (p < 0) continue;
      if constexpr (CODES) {
        // the largest scale of the place's block
        const int b0 = row >> a.s.shift << a.s.shift, b1 = min(n, b0 + (1 << a.s.shift));
        float now = 0.f;
        for (int k = b0; k < b1; ++k) now = fmaxf(now, s_was[k]);
        const float was = s_was[row];
        if (was != now) {
          float y[16];
          codes_float<C>(x[i], y);
          x[i] = to_codes16<C>(y, now > 0.f ? was / now : 0.f);
        }
        if (row == b0 && at == row * vecs)
          scale[p * a.s.page + (((j0 + row) & slots) >> a.s.shift) * a.s.block] = now;
      }
      *reinterpret_cast<uint4*>(data + p * c.page_b + ((j0 + row) & slots) * c.slot_b +
                                16 * (at - row * vecs)) = x[i];
    }
    if constexpr (CODES) __syncthreads();
  }
}

}  // namespace

size_t cache_evict_workspace(const CacheView& c, int64_t) {
  return sls_align256((size_t)c.B * 4);
}

int launch_cache_evict(const EvictArgs& a, int code, void* workspace, cudaStream_t stream) {
  const CacheView& c = a.c;
  if (c.B == 0) return SLS_OK;
  if ((int64_t)c.B * c.kv_heads * 2 * EV_CLUSTER > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  int32_t* lens = (int32_t*)workspace;
  int st = at_launch(cache_evict_select_kernel, dim3((unsigned)(c.B * c.kv_heads)), EV_T, 0, 1,
                     stream, a, lens);
  if (st != SLS_OK) return st;
  // no more CTAs of a cluster than waves have rows for
  int cluster = 1;
  while (cluster < EV_CLUSTER && cluster * EV_ROWS < a.keep) cluster *= 2;
  const dim3 grid((unsigned)(c.B * c.kv_heads * 2 * cluster));
  auto kern = code == SLS_I8     ? cache_evict_move_kernel<I8>
              : code == SLS_E4M3 ? cache_evict_move_kernel<E4M3>
                                 : cache_evict_move_kernel<void>;
  return at_launch(kern, grid, EV_MOVE_T, 0, cluster, stream, a, lens);
}

}  // namespace sls
