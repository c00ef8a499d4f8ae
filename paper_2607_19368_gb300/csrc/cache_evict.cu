// Eviction: of every (sequence, key head) the first and last tokens and the heaviest others
// stay, in order, and move to the front of the sequence's pages.
//
// Two launches.  The first selects: a cluster holds a sequence's weights in shared memory, finds
// that of the last of the kept others digit by digit (counts of 2048, 2048 and 1024 digits of the
// weights as ordered integers, summed through distributed shared memory), and counts what stays in
// front of every token, which gives it its place; weights move here.  The second moves keys and values.  A place is never behind its source, so a cluster of
// CTAs takes the places in waves, in order: what a wave reads lies at or behind its first place,
// what earlier waves wrote lies in front of it, and the one barrier between a wave's reads and its
// writes is all that moving in place needs.
//
// Bound by the bytes of weights and moved rows in the limit, here by latency: a selection is a
// chain of a dozen barriers over a cluster, a wave one of dependent loads (index, page, row) and a
// barrier.  One prompt of 32768 tokens to 2048, 4 heads of 128, bfloat16: 20 us; 24 of up to 8192 to
// 1024, 8 heads, e4m3: 38 us, of it 22 and 24 under a profiler for the two launches, which overlap.
#include <algorithm>

#include "cache8.cuh"

namespace sls {

namespace {

constexpr int EV_T = 512;     // selection
constexpr int EV_PER = 4;     // digits that a thread counts up: EV_BINS / EV_T
constexpr int EV_BINS = 2048;
constexpr int EV_ROOM = 12288;  // groups of four weights that a CTA of the selection holds at most
constexpr int EV_MOVE_T = 256;
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

SLS_DEV void ev_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// What a CTA of the selection has in shared memory.
struct __align__(16) EvShared {
  unsigned bins[2][EV_BINS];
  unsigned warp[EV_T / 32][2];
  unsigned total[EV_CLUSTER];  // of the cluster's CTAs: staying ones, equal ones
  unsigned digit, above, count;  // a pass's digit, how many are above it and have it
};

// The digit of this pass at which the count from the top reaches `need`, from a thread's counts:
// n[i] of digit ev_first() + i.
SLS_DEV int ev_first() { return EV_BINS - EV_PER - EV_PER * (int)threadIdx.x; }
SLS_DEV void ev_digit(EvShared& s, const unsigned (&n)[EV_PER], unsigned need) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned own = 0;
#pragma unroll
  for (int i = 0; i < EV_PER; ++i) own += n[i];
  unsigned sum = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 31) s.warp[warp][0] = sum;
  __syncthreads();
  unsigned above = lane < warp ? s.warp[lane][0] : 0u;
  above = __reduce_add_sync(0xffffffffu, above) + sum - own;
#pragma unroll
  for (int i = EV_PER - 1; i >= 0; --i) {
    if (above < need && need <= above + n[i])
      s.digit = ev_first() + i, s.above = above, s.count = n[i];
    above += n[i];
  }
  __syncthreads();
}

SLS_DEV int ev_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
SLS_DEV uint32_t ev_digits(int pass) { return pass == 2 ? 1023u : 2047u; }

// The selection by one CTA that reads the weights anew for every pass: any length.
SLS_DEV void ev_select_long(const EvictArgs& a, const EvSeq& e, int len, int32_t* kept, EvShared& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = a.first, hi = len - a.last;
  unsigned need = (unsigned)(a.keep - a.first - a.last);
  uint32_t top = 0, mask = 0;
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int shift = ev_shift(pass);
    const uint32_t digits = ev_digits(pass);
    unsigned* bins = s.bins[0];
    for (int i = threadIdx.x; i < EV_BINS; i += EV_T) bins[i] = 0;
    __syncthreads();
    for (int x0 = lo; x0 < hi; x0 += EV_T) {
      const int x = x0 + threadIdx.x;
      const float* w = x < hi ? e.weight(x) : nullptr;
      const uint32_t k = ev_key(w ? *w : 0.f);
      if (x < hi && (k & mask) == top) atomicAdd(&bins[(k >> shift) & digits], 1u);
    }
    __syncthreads();
    unsigned n[EV_PER];
#pragma unroll
    for (int i = 0; i < EV_PER; ++i) n[i] = bins[ev_first() + i];
    ev_digit(s, n, need);
    top |= s.digit << shift;
    mask |= digits << shift;
    need -= s.above;
    const bool all = need == s.count;  // all that share these digits stay
    __syncthreads();
    if (all) break;
  }
  // in order: larger ones and the first `need` equal ones stay
  unsigned base_more = 0, base_same = 0;
  for (int x0 = 0; x0 < len; x0 += EV_T) {
    const int x = x0 + threadIdx.x;
    float w = 0.f;
    bool more = false, same = false;
    if (x < len) {
      const float* p = e.weight(x);
      w = p ? *p : 0.f;
      const uint32_t k = ev_key(w);
      more = x < lo || x >= hi || (k & mask) > top;
      same = !more && mask != 0 && (k & mask) == top;
    }
    const unsigned bm = __ballot_sync(0xffffffffu, more), bs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) s.warp[warp][0] = __popc(bm), s.warp[warp][1] = __popc(bs);
    __syncthreads();  // the tile's weights are read, too
    const unsigned low = (1u << lane) - 1;
    unsigned m = base_more + __popc(bm & low), q = base_same + __popc(bs & low);
    for (int v = 0; v < EV_T / 32; ++v) {
      if (v < warp) m += s.warp[v][0], q += s.warp[v][1];
      base_more += s.warp[v][0], base_same += s.warp[v][1];
    }
    if (more || (same && q < need)) {
      const unsigned to = m + min(q, need);
      kept[to] = x;
      if (to != (unsigned)x)
        if (float* p = e.weight(to)) *p = w;
    }
    __syncthreads();
  }
  for (int x = a.keep + threadIdx.x; x < len; x += EV_T)
    if (float* p = e.weight(x)) *p = 0.f;
}

__global__ void __launch_bounds__(EV_T, 2)
cache_evict_select_kernel(const __grid_constant__ EvictArgs a, int room4) {
  extern __shared__ float4 s_w[];  // room4 of them
  __shared__ EvShared s;
  const CacheView& c = a.c;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int unit = blockIdx.x / size;
  const int seq = unit / c.kv_heads, h = unit - seq * c.kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < 2 * EV_BINS; i += EV_T) s.bins[0][i] = 0;
  at_go();
  at_wait_ahead();
  const int len = (int)cache_len(c, seq);
  int32_t* kept = a.kept + ((int64_t)seq * c.kv_heads + h) * a.keep;
  const EvSeq e{a, seq, h};
  if (len <= a.keep) {
    for (int64_t i = rank * EV_T + threadIdx.x; i < a.keep; i += size * EV_T)
      kept[i] = i < len ? (int)i : -1;
    return;
  }
  // this CTA's weights, four in a row at a time, to shared memory: loops over them stay short, and
  // nearly all of the time of a call this small goes into fetching its instructions
  const int groups = (len + 3) >> 2, per = (groups + size - 1) / size;
  if (per > room4) {
    if (rank == 0) ev_select_long(a, e, len, kept, s);
    return;
  }
  const int g0 = min(groups, (int)rank * per), mine = min(groups, g0 + per) - g0;
#pragma unroll 4
  for (int g = threadIdx.x; g < mine; g += EV_T) {
    const float* p = e.weight(4 * (int64_t)(g0 + g));
    s_w[g] = p ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const int lo = a.first, hi = len - a.last;
  unsigned need = (unsigned)(a.keep - a.first - a.last);
  uint32_t top = 0, mask = 0;
  __syncthreads();
  // Another CTA's shared memory may be written once that CTA runs: a digit's barrier says so, and where
  // the first and last tokens are all that stays this one.
  if (need == 0) ev_cluster_sync();
#pragma unroll 1
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int shift = ev_shift(pass);
    const uint32_t digits = ev_digits(pass);
    unsigned* bins = s.bins[pass & 1];
#pragma unroll 1
    for (int g = threadIdx.x; g < mine; g += EV_T) {
      const float4 f = s_w[g];
      const float w[4] = {f.x, f.y, f.z, f.w};
      const int x = 4 * (g0 + g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t k = ev_key(w[i]);
        if (x + i >= lo && x + i < hi && (k & mask) == top)
          atomicAdd(&bins[(k >> shift) & digits], 1u);
      }
    }
    ev_cluster_sync();
    // of all CTAs of the cluster
    unsigned n[EV_PER] = {};
#pragma unroll 4
    for (uint32_t r = 0; r < size; ++r) {
      uint32_t at;
      unsigned x[EV_PER];
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&bins[ev_first()])), "r"(r));
      asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                   : "r"(at)
                   : "memory");
#pragma unroll
      for (int i = 0; i < EV_PER; ++i) n[i] += x[i];
    }
    // nobody reads the first pass's counts any more when the second pass's are complete
    if (pass == 1)
      for (int i = threadIdx.x; i < EV_BINS; i += EV_T) s.bins[0][i] = 0;
    ev_digit(s, n, need);
    top |= s.digit << shift;
    mask |= digits << shift;
    need -= s.above;
    if (need == s.count) break;  // all that share these digits stay
    __syncthreads();
  }
  // ---- places: larger ones and the first `need` equal ones stay, in order.  A thread has groups
  // in a row; counts hold what stays in their low half and what is equal in their high half (at most
  // 49152 a CTA).
  auto kind = [&](int x, float f) {
    const uint32_t k = ev_key(f);
    if (x >= len) return 0u;
    if (x < lo || x >= hi || (k & mask) > top) return 1u;
    return mask != 0 && (k & mask) == top ? 1u << 16 : 0u;
  };
  const int q = (mine + EV_T - 1) / EV_T, first = min(mine, (int)threadIdx.x * q),
            last = min(mine, first + q);
  unsigned own = 0;
#pragma unroll 1
  for (int g = first; g < last; ++g) {
    const float4 f = s_w[g];
    const int x = 4 * (g0 + g);
    own += kind(x, f.x) + kind(x + 1, f.y) + kind(x + 2, f.z) + kind(x + 3, f.w);
  }
  unsigned sum = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 31) s.warp[warp][1] = sum;
  __syncthreads();
  const unsigned each = lane < EV_T / 32 ? s.warp[lane][1] : 0u;
  const unsigned total = __reduce_add_sync(0xffffffffu, each);
  unsigned base = __reduce_add_sync(0xffffffffu, lane < warp ? each : 0u) + sum - own;
  if (warp == 0 && lane < size) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&s.total[rank])), "r"(lane));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(total) : "memory");
  }
  // all weights of the sequence are in shared memory, all totals known; nobody touches another
  // CTA's shared memory after this
  ev_cluster_sync();
  unsigned more = base & 0xffffu, same = base >> 16;
  for (uint32_t r = 0; r < rank; ++r) more += s.total[r] & 0xffffu, same += s.total[r] >> 16;
#pragma unroll 1
  for (int g = first; g < last; ++g) {
    const float4 f = s_w[g];
    const float w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = 4 * (g0 + g) + i;
      const unsigned k = kind(x, w[i]);
      if (k == 1 || (k > 1 && same < need)) {
        const unsigned to = more + min(same, need);
        kept[to] = x;
        if (to != (unsigned)x)
          if (float* p = e.weight(to)) *p = w[i];
      }
      more += k & 1, same += k >> 16;
    }
  }
  // four slots at a time from the first multiple of four on
  const int64_t z0 = ((int64_t)a.keep + 3) & ~(int64_t)3;
  for (int x = a.keep + threadIdx.x; x < min(z0, (int64_t)len) && rank == 0; x += EV_T)
    if (float* p = e.weight(x)) *p = 0.f;
#pragma unroll 1
  for (int64_t x = z0 + 4 * (int64_t)(rank * EV_T + threadIdx.x); x < len; x += 4 * size * EV_T)
    if (float* p = e.weight(x)) {
      if (x + 4 <= len) *reinterpret_cast<float4*>(p) = make_float4(0.f, 0.f, 0.f, 0.f);
      else
        for (int i = 0; x + i < len; ++i) p[i] = 0.f;
    }
}

// C: I8 or E4M3, or void for 16-bit elements; BOTH: a cluster moves keys and values, which
// share their places, else one of them.
template <typename C, bool BOTH>
struct EvMove {
  static constexpr bool CODES = !std::is_void<C>::value;
  static constexpr int ROWS = CODES || !BOTH ? 128 : 64;  // of a CTA's wave: whole blocks of codes
  static constexpr int MATS = BOTH ? 2 : 1;
  // vectors of 16 bytes of a thread for each of them
  static constexpr int V = ROWS * SLS_MAX_HEAD_DIM * (CODES ? 1 : 2) / 16 / EV_MOVE_T;
};

template <typename C, bool BOTH>
__global__ void __launch_bounds__(EV_MOVE_T, 4)
cache_evict_move_kernel(const __grid_constant__ EvictArgs a) {
  using S = EvMove<C, BOTH>;
  __shared__ int64_t s_from[S::ROWS], s_to[S::ROWS];  // byte offsets of rows, or -1
  __shared__ float s_was[S::MATS][S::ROWS], s_by[S::MATS][S::ROWS];  // codes: old scale, old / new
  const CacheView& c = a.c;
  uint32_t rank, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int unit = blockIdx.x / size;
  const int heads = BOTH ? c.kv_heads : 2 * c.kv_heads;
  const int seq = unit / heads, hk = unit - seq * heads;
  const int h = hk % c.kv_heads;
  at_go();
  at_wait_ahead();
  // the one reader of a length here cuts it
  if (hk == 0 && rank == 0 && threadIdx.x == 0 && cache_len(c, seq) > a.keep) a.lens[seq] = a.keep;
  const int32_t* kept = a.kept + ((int64_t)seq * c.kv_heads + h) * a.keep;
  // kept indices rise: where the last one is in its place all are, and -1 ends a shorter sequence
  if (a.keep == 0 || kept[a.keep - 1] < a.keep) return;  // the whole cluster
  const int32_t* table = c.table + seq * c.table_ld;
  const bool values = !BOTH && hk >= c.kv_heads;
  char* const mat[2] = {values ? c.v : c.k, c.v};
  float* const scale[2] = {(values ? a.s.v : a.s.k) + h * a.s.head, a.s.v + h * a.s.head};
  const int vecs = c.head_dim * (S::CODES ? 1 : 2) / 16;
  const int slots = (1 << c.page_shift) - 1;
  for (int w0 = 0; w0 < a.keep; w0 += S::ROWS * (int)size) {
    const int j0 = w0 + (int)rank * S::ROWS;
    const int n = min(S::ROWS, a.keep - j0);
    if ((int)threadIdx.x < n) {
      const int to = j0 + threadIdx.x, from = kept[to];
      const int64_t p = table[from >> c.page_shift], q = table[to >> c.page_shift];
      const bool real = p >= 0 && p < c.num_pages;
      s_from[threadIdx.x] = real ? p * c.page_b + (from & slots) * c.slot_b + h * c.head_b : -1;
      s_to[threadIdx.x] = q >= 0 && q < c.num_pages
                              ? q * c.page_b + (to & slots) * c.slot_b + h * c.head_b
                              : -1;
      if constexpr (S::CODES)
#pragma unroll
        for (int m = 0; m < S::MATS; ++m)
          s_was[m][threadIdx.x] =
              real ? scale[m][p * a.s.page + ((from & slots) >> a.s.shift) * a.s.block] : 0.f;
    }
    __syncthreads();
    uint4 x[S::MATS][S::V];
#pragma unroll
    for (int i = 0; i < S::V; ++i) {
      const int at = i * EV_MOVE_T + threadIdx.x, row = at / vecs;
#pragma unroll
      for (int m = 0; m < S::MATS; ++m) x[m][i] = make_uint4(0, 0, 0, 0);
      if (row >= n) continue;
      const int64_t from = s_from[row];
      if (from >= 0)
#pragma unroll
        for (int m = 0; m < S::MATS; ++m)
          x[m][i] = *reinterpret_cast<const uint4*>(mat[m] + from + 16 * (at - row * vecs));
    }
    float now[S::MATS];  // codes: of thread `row`'s block, the size of the largest scale that its rows come from
    if constexpr (S::CODES) {
      const int row = threadIdx.x;
      if (row < n) {
        const int b0 = row >> a.s.shift << a.s.shift, b1 = min(n, b0 + (1 << a.s.shift));
#pragma unroll
        for (int m = 0; m < S::MATS; ++m) {
          now[m] = 0.f;
          for (int k = b0; k < b1; ++k) now[m] = fmaxf(now[m], fabsf(s_was[m][k]));
          const float was = s_was[m][row];
          s_by[m][row] = was == now[m] ? 1.f : now[m] > 0.f ? was / now[m] : 0.f;
        }
      }
    }
    ev_cluster_sync();
    if constexpr (S::CODES) {
      const int row = threadIdx.x;
      if (row < n && (row & ((1 << a.s.shift) - 1)) == 0 && s_to[row] >= 0) {
        const int64_t q = table[(j0 + row) >> c.page_shift];
#pragma unroll
        for (int m = 0; m < S::MATS; ++m)
          scale[m][q * a.s.page + (((j0 + row) & slots) >> a.s.shift) * a.s.block] = now[m];
      }
    }
#pragma unroll
    for (int i = 0; i < S::V; ++i) {
      const int at = i * EV_MOVE_T + threadIdx.x, row = at / vecs;
      if (row >= n) continue;
      const int64_t to = s_to[row];
      if (to < 0) continue;
#pragma unroll
      for (int m = 0; m < S::MATS; ++m) {
        if constexpr (S::CODES) {
          const float by = s_by[m][row];
          if (by != 1.f) {
            float y[16];
            codes_float<C>(x[m][i], y);
            x[m][i] = to_codes16<C>(y, by);
          }
        }
        *reinterpret_cast<uint4*>(mat[m] + to + 16 * (at - row * vecs)) = x[m][i];
      }
    }
    __syncthreads();
  }
}

template <typename C>
int launch_move(const EvictArgs& a, int sms, cudaStream_t stream) {
  const CacheView& c = a.c;
  // keys and values by one cluster where there are clusters enough without (sequences to 8192, 8 heads
  // of 128 in e4m3, to 1024: 4 of them 17.8 us so, 17.5 apart; 6 21.4 and 23.3; 12 29.8 and 32.0)
  const int64_t units = (int64_t)c.B * c.kv_heads;
  const bool both = units * EV_CLUSTER >= 2 * sms;
  const int rows = both ? EvMove<C, true>::ROWS : EvMove<C, false>::ROWS;
  int cluster = 1;  // no more CTAs than waves have rows for
  while (cluster < EV_CLUSTER && cluster * rows < a.keep) cluster *= 2;
  const dim3 grid((unsigned)(units * (both ? 1 : 2) * cluster));
  return at_launch(both ? cache_evict_move_kernel<C, true> : cache_evict_move_kernel<C, false>,
                   grid, EV_MOVE_T, 0, cluster, stream, a);
}

}  // namespace

int launch_cache_evict(const EvictArgs& a, int code, cudaStream_t stream) {
  const CacheView& c = a.c;
  if (c.B == 0) return SLS_OK;
  if ((int64_t)c.B * c.kv_heads * 2 * EV_CLUSTER > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  static int sm_count[64] = {};  // per device
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  int sms = dev < 64 ? sm_count[dev] : 0;
  if (sms == 0) {
    SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    SLS_CUDA_TRY(cudaFuncSetAttribute(cache_evict_select_kernel,
                                      cudaFuncAttributeMaxDynamicSharedMemorySize, EV_ROOM * 16));
    if (dev < 64) sm_count[dev] = sms;
  }
  // CTAs of a selection: as many as share out the GPU, no more than give every thread four weights
  // of the longest table, and enough to hold it (past 8 x 49152 tokens one CTA reads it anew each
  // pass)
  const int64_t room = (int64_t)c.max_pages << c.page_shift, units = (int64_t)c.B * c.kv_heads;
  int size = 1;
  while (size < EV_CLUSTER && ((units * size <= sms && size * EV_T * 4 < room) ||
                               (int64_t)size * EV_ROOM * 4 < room))
    size *= 2;
  const int room4 = (int)std::min<int64_t>(EV_ROOM, ((room + 3) / 4 + size - 1) / size);
  int st = at_launch(cache_evict_select_kernel, dim3((unsigned)(units * size)), EV_T,
                     (size_t)room4 * 16, size, stream, a, room4);
  if (st != SLS_OK) return st;
  return code == SLS_I8     ? launch_move<I8>(a, sms, stream)
         : code == SLS_E4M3 ? launch_move<E4M3>(a, sms, stream)
                            : launch_move<void>(a, sms, stream);
}

}  // namespace sls
