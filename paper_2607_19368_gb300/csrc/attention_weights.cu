// The weight that queries place on every cached token, summed over rows i (tokens) and the
// query heads of a key head and added to a running sum:
//   w_j += sum_i exp(s_ij - m_i) / l_i,   m_i = max_j s_ij,  l_i = sum_j exp(s_ij - m_i).
//
// A column can be summed only when the rows' m and l are known, so there are two passes over
// the scores, both on the tensor cores in 128 x 128 tiles.  The first has rows as the lanes of
// tensor memory, so that a thread finds the maximum and sum of a row's 64 tokens by itself; a
// small launch joins the pieces of rows.  The second has tokens as lanes: a thread adds up a
// token's column, with the rows' maxima and sums read from shared memory by all at once.  No sum is
// made by atomics: the same call gives the same bits.
//
// An exponent is one multiply-add of the score, with the row's maximum times the scale, rounded, as
// the summand; what that rounding is off by, the same for all of a row, is taken out of its
// sum and of the factor of its weights (left in, it is 2^-24 of the maximum's exponent: 1.4e-6 of the
// weights instead of 2e-7 where scores reach 30).
//
// Bound by exponentials (two a score) and, for few rows, by the products of padded tiles; the keys'
// bytes are below either from some ten rows on.  A CTA goes through phases in step (keys to shared
// memory, codes to float16 on the way; products; scores), with the next keys on their way in
// registers; two CTAs an SM fill each other's gaps.  32 rows (tokens) of 7 heads over 32768
// tokens of 4 key heads, e4m3: 57.8 us, 24.0 the first pass and 34.5 the second (86 us with mma.sync,
// whose products took the time); 58.7 million exponentials are 12 us at 16 a cycle and SM.  A CTA has
// 7 tiles of a row tile, then 3.4 units of two: in a trace 9000 to 15000 of its 36000 and 46000
// cycles go until the first scores (lengths, pages, rows), a tile's scores take 1700 to 2400.
//
// Where rows are few (a token for each sequence) the kernels of attention_weights_few.cu read keys
// once instead.
#include <algorithm>

#include "attention_decode.cuh"
#include "attention_umma.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int AW_T = 256;
constexpr int AW_TILE = 128;  // rows or tokens
constexpr int AW_JOIN_WARPS = 8;

struct AwPlan {
  int group;        // query heads of a key head
  int ctas;         // of the first pass: most parts
  int64_t* prefix;  // B + 1: first-pass steps before every sequence
  float2* ml;       // (part, first or last piece, row of a tile): maximum and sum
  float2* stat;     // (token, query head): maximum, sum; then what makes the weight of a score
};

// KT: element of keys (E, or codes)
template <typename E, typename KT, int HD>
struct AwShape {
  static constexpr bool CODES = !std::is_same<E, KT>::value;
  using M = typename std::conditional<CODES, __half, E>::type;  // of the products
  static constexpr int HALF_BYTES = AW_TILE * 128;
  static constexpr int TILE_BYTES = HD / 64 * HALF_BYTES;
  static constexpr int KEY_LANES = HD / (CODES ? 16 : 8);       // threads of a key's row
  static constexpr int KEY_LOADS = AW_TILE * KEY_LANES / AW_T;  // 16-byte loads of a thread
  static constexpr int ROW_LANES = HD / 8;
  static constexpr int ROW_LOADS = AW_TILE * ROW_LANES / AW_T;
  static constexpr uint32_t FMT = std::is_same<M, __nv_bfloat16>::value ? 1u : 0u;
  static constexpr uint32_t IDESC = (1u << 4) | (FMT << 7) | (FMT << 10) |
                                    ((uint32_t)(AW_TILE >> 4) << 24) |
                                    ((uint32_t)(AW_TILE >> 3) << 17);
  // Byte of 16-byte chunk ch of a row of a tile.
  SLS_DEV static int at(int row, int ch) {
    return (ch >> 3) * HALF_BYTES + row * 128 + (((ch & 7) ^ (row & 7)) << 4);
  }
};

// The packed rows of a sequence.
SLS_DEV void aw_tokens(const AttnArgs& a, int seq, int64_t& q0, int64_t& q1) {
  if (a.cu) seq_rows(a.cu, seq, a.T, q0, q1);
  else q0 = seq, q1 = seq + 1;
}

SLS_DEV int64_t aw_row_tiles(const AttnArgs& a, int group, int seq) {
  int64_t q0, q1;
  aw_tokens(a, seq, q0, q1);
  return ((q1 - q0) * group + AW_TILE - 1) >> 7;
}

// A key head of a sequence.
struct AwHead {
  int seq, h, len, n, group;
  int64_t q0, rows;
  SLS_DEV AwHead(const AttnArgs& a, int g, int s, int head) : seq(s), h(head), group(g) {
    len = (int)cache_len(a.c, s);
    int64_t q1;
    aw_tokens(a, s, q0, q1);
    n = (int)(q1 - q0);
    rows = (int64_t)n * group;
  }
};

// A tile of its rows.
struct AwRows {
  int count;     // rows of the tile
  int tok, rem;  // the first row's token, and which of its query heads
  int mul;       // x / group = x * mul >> 16 for x < 256
  SLS_DEV AwRows(const AwHead& w, int64_t tile) {
    const int64_t base = tile * AW_TILE;
    count = (int)max((int64_t)0, min((int64_t)AW_TILE, w.rows - base));
    tok = (int)ad_div(base, w.group);
    rem = (int)(base - (int64_t)tok * w.group);
    mul = (65536 + w.group - 1) / w.group;
  }
  // token and query head of row r of the tile
  SLS_DEV int token(int r, const AwHead& w, int& g) const {
    const int d = ((rem + r) * mul) >> 16;
    g = rem + r - d * w.group;
    return tok + d;
  }
  // tokens of the cache that it sees
  SLS_DEV int see(const AttnArgs& a, const AwHead& w, int r) const {
    int g;
    return r >= count ? 0 : a.causal ? max(0, w.len - w.n + token(r, w, g) + 1) : w.len;
  }
  // its (token, query head) among all
  SLS_DEV int64_t packed(const AttnArgs& a, const AwHead& w, int r) const {
    int g;
    const int t = token(r, w, g);
    return (w.q0 + t) * a.q_heads + w.h * w.group + g;
  }
};

// 128 keys from token key0 on: their pages, then the keys, to registers, and from there to a tile.
// Page numbers are fetched a tile ahead, so that keys are one latency away.
template <typename E, typename KT, int HD>
struct AwKeys {
  using S = AwShape<E, KT, HD>;
  uint4 raw[S::KEY_LOADS];
  int page[S::KEY_LOADS], own;  // of the keys to load next (-1: none), and that of key threadIdx.x
  float scale;                  // of key threadIdx.x

  SLS_DEV void pages(const AttnArgs& a, const AwHead& w, int key0) {
    const CacheView& c = a.c;
    const int32_t* table = c.table + w.seq * c.table_ld;
    const bool on = threadIdx.x % S::KEY_LANES * (S::CODES ? 16 : 8) < c.head_dim;
#pragma unroll
    for (int i = 0; i < S::KEY_LOADS; ++i) {
      const int x = key0 + i * (AW_T / S::KEY_LANES) + threadIdx.x / S::KEY_LANES;
      page[i] = on && x < w.len ? table[x >> c.page_shift] : -1;
    }
    const int x = key0 + threadIdx.x;
    own = S::CODES && threadIdx.x < AW_TILE && x < w.len ? table[x >> c.page_shift] : -1;
  }
  SLS_DEV void load(const AttnArgs& a, const ScaleView& sc, const AwHead& w, int key0) {
    const CacheView& c = a.c;
    const int slots = (1 << c.page_shift) - 1;
    const char* base = c.k + w.h * c.head_b + 16 * (threadIdx.x % S::KEY_LANES);
#pragma unroll
    for (int i = 0; i < S::KEY_LOADS; ++i) {
      const int x = key0 + i * (AW_T / S::KEY_LANES) + threadIdx.x / S::KEY_LANES;
      raw[i] = make_uint4(0, 0, 0, 0);
      if (page[i] >= 0 && page[i] < c.num_pages)
        raw[i] = *reinterpret_cast<const uint4*>(base + page[i] * c.page_b + (x & slots) * c.slot_b);
    }
    if constexpr (S::CODES) {
      scale = 0.f;
      const int x = key0 + threadIdx.x;
      if (own >= 0 && own < c.num_pages)
        scale = sc.k[own * sc.page + ((x & slots) >> sc.shift) * sc.block + w.h * sc.head];
    }
  }

  SLS_DEV void store(unsigned char* tile, float* scales) const {
    const int ch = threadIdx.x % S::KEY_LANES;
#pragma unroll
    for (int i = 0; i < S::KEY_LOADS; ++i) {
      const int row = i * (AW_T / S::KEY_LANES) + threadIdx.x / S::KEY_LANES;
      if constexpr (S::CODES) {
        uint4 y, z;
        codes_half<KT>(raw[i].x, y.x, y.y);
        codes_half<KT>(raw[i].y, y.z, y.w);
        codes_half<KT>(raw[i].z, z.x, z.y);
        codes_half<KT>(raw[i].w, z.z, z.w);
        *reinterpret_cast<uint4*>(tile + S::at(row, 2 * ch)) = y;
        *reinterpret_cast<uint4*>(tile + S::at(row, 2 * ch + 1)) = z;
      } else {
        *reinterpret_cast<uint4*>(tile + S::at(row, ch)) = raw[i];
      }
    }
    if constexpr (S::CODES)
      if (threadIdx.x < AW_TILE) scales[threadIdx.x] = scale;
  }
};

// A tile of rows to shared memory; factors (codes with bfloat16 queries: a row's power of two, as in
// the decode kernel) to `factor`.
template <typename E, typename KT, int HD>
SLS_DEV void aw_stage_rows(const AttnArgs& a, const AwHead& w, const AwRows& rows,
                           unsigned char* out, float* factor) {
  using S = AwShape<E, KT, HD>;
  const int ch = threadIdx.x % S::ROW_LANES;
  uint4 all[S::ROW_LOADS];
#pragma unroll
  for (int i = 0; i < S::ROW_LOADS; ++i) {
    const int r = i * (AW_T / S::ROW_LANES) + threadIdx.x / S::ROW_LANES;
    all[i] = make_uint4(0, 0, 0, 0);
    if (r < rows.count && 8 * ch < a.c.head_dim) {
      int g;
      const int tok = rows.token(r, w, g);
      all[i] = *reinterpret_cast<const uint4*>(a.q.data + (w.q0 + tok) * a.q.token_b +
                                               (w.h * w.group + g) * a.q.head_b + 16 * ch);
    }
  }
#pragma unroll
  for (int i = 0; i < S::ROW_LOADS; ++i) {
    const int r = i * (AW_T / S::ROW_LANES) + threadIdx.x / S::ROW_LANES;
    uint4 u = all[i];
    float back = 1.f;
    if constexpr (!std::is_same<E, typename S::M>::value) {
      float x[8], top = 0.f;
      widen8<E>(u, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
      for (int d = 1; d < S::ROW_LANES; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      // the largest element to [2^14, 2^15)
      const int e = max(__float_as_int(top) >> 23, 16);
      const float by = __int_as_float((127 + 14 + 127 - e) << 23);
      back = __int_as_float((e - 14) << 23);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= by;
      u = narrow8<__half>(x);
    }
    *reinterpret_cast<uint4*>(out + S::at(r, ch)) = u;
    if (ch == 0) factor[r] = back;
  }
}

// D = A B^T of two tiles, to tensor memory columns d on; commits to `bar`.
template <typename E, typename KT, int HD>
SLS_DEV void aw_products(uint32_t lead, uint32_t d, const unsigned char* a, const unsigned char* b,
                         uint64_t* bar) {
  using S = AwShape<E, KT, HD>;
  const uint32_t ad = ap_desc(smem_u32(a), 16), bd = ap_desc(smem_u32(b), 16);
#pragma unroll
  for (int k = 0; k < HD / 16; ++k) {
    const uint32_t off = ((k >> 2) * S::HALF_BYTES + (k & 3) * 32) >> 4;
    ap_mma_ss(lead, d, ad + off, bd + off, S::IDESC, k > 0);
  }
  ap_commit(lead, bar);
}

// Writes to shared memory are seen by the tensor cores after this and a barrier.
SLS_DEV void aw_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int COLUMNS>
SLS_DEV uint32_t aw_alloc(uint32_t* holder) {
  if (threadIdx.x < 32) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(holder)),
                 "r"(COLUMNS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  ap_fence_before();
  __syncthreads();
  ap_fence_after();
  return *holder;
}
template <int COLUMNS>
SLS_DEV void aw_free(uint32_t tmem) {
  ap_fence_before();
  __syncthreads();
  if (threadIdx.x < 32) {
    ap_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLUMNS)
                 : "memory");
  }
}

// A sum of 2^(v f + off), off the rounded -m f, as that of 2^((v - m) f): the rounding's remainder x is
// exact by one multiply-add and far below 1, 2^-x to first order.
SLS_DEV float aw_exact(float sum, float m, float f, float off) {
  return __fmaf_rn(sum, -0.69314718f * __fmaf_rn(m, f, off), sum);
}

// ---- first pass: maxima and sums of rows -------------------------------------------------
template <typename E, typename KT, int HD>
__global__ void __launch_bounds__(AW_T, 2)
attention_weights_rows_kernel(const __grid_constant__ AttnArgs a,
                              const __grid_constant__ ScaleView sc, const __grid_constant__ AwPlan p,
                              int* status) {
  using S = AwShape<E, KT, HD>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ int64_t s_pre[AW_T + 1];
  __shared__ float s_factor[AW_TILE];
  // of four tiles: a thread may fetch two ahead of one that still reads
  __shared__ __align__(16) float s_scale[4][AW_TILE];
  __shared__ float2 s_ml[AW_TILE];
  __shared__ uint64_t bar[2];
  __shared__ uint32_t holder;
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float cs = a.scale * 1.4426950408889634f;
  unsigned char* rows_s = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* keys_s = rows_s + S::TILE_BYTES;

  at_wait_ahead();
  if (threadIdx.x < 2) mbar_init(&bar[threadIdx.x], 1);
  mbar_fence_init();
  const auto steps = [&](int s) {
    return (int64_t)ad_steps<AW_TILE>(c, s) * aw_row_tiles(a, p.group, s) * c.kv_heads;
  };
  const int R = ad_prefix<AW_T>(c, s_pre, p.prefix, steps);
  const int64_t total = s_pre[AW_T];
  const int parts = (int)min((int64_t)p.ctas, total);
  if ((int)blockIdx.x >= parts) return;
  const int64_t t0 = ad_div(total * blockIdx.x, parts), t1 = ad_div(total * (blockIdx.x + 1), parts);
  const uint32_t tmem = aw_alloc<2 * AW_TILE>(&holder);
  const uint32_t lead = at_elect();
  int seq;
  int64_t before;  // steps before seq
  ad_find<AW_T>(s_pre, R, t0, steps, seq, before);
  // this thread's row of a tile, and its columns
  const int r = 32 * (warp & 3) + lane, col0 = 64 * (warp >> 2);
  const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + col0;
  unsigned turn = 0;  // tiles of keys so far: they take turns at memory, columns and barriers
  bool ok = true;

  int64_t t = t0;
  while (t < t1 && ok) {
    // ---- a piece: key tiles [j0, j1) of a tile of rows ----
    const int64_t all = steps(seq);
    if (t - before >= all) {
      before += all;
      ++seq;
      continue;
    }
    const int n = ad_steps<AW_TILE>(c, seq);
    const int64_t item = ad_div(t - before, n), tiles = aw_row_tiles(a, p.group, seq);
    const int j0 = (int)(t - before - item * n), j1 = (int)min((int64_t)n, j0 + t1 - t);
    const int h = (int)ad_div(item, tiles);
    const AwHead w(a, p.group, seq, h);
    const AwRows rows(w, item - h * tiles);
    AwKeys<E, KT, HD> keys;
    keys.pages(a, w, j0 * AW_TILE);
    aw_stage_rows<E, KT, HD>(a, w, rows, rows_s, s_factor);
    const int see = rows.see(a, w, r);
    // tokens that the last row sees, and so any
    const int last = min(j1, (rows.see(a, w, rows.count - 1) + AW_TILE - 1) / AW_TILE);
    float m = -INFINITY, l = 0.f;
    // products of the next tile run while the scores of one are worked on
    auto next = [&](int j, unsigned k) {
      keys.store(keys_s + (k & 1) * S::TILE_BYTES, s_scale[k & 3]);
      aw_fence();
      __syncthreads();  // and the scores that were in these columns are read
      if (warp == 0) {
        ap_fence_after();
        aw_products<E, KT, HD>(lead, tmem + (k & 1) * AW_TILE, rows_s, keys_s + (k & 1) * S::TILE_BYTES,
                               &bar[k & 1]);
      }
      if (j + 1 < last) keys.load(a, sc, w, (j + 1) * AW_TILE);
      if (j + 2 < last) keys.pages(a, w, (j + 2) * AW_TILE);
    };
    if (j0 < last) {
      keys.load(a, sc, w, j0 * AW_TILE);
      keys.pages(a, w, (j0 + 1) * AW_TILE);
      next(j0, turn);
    } else {
      __syncthreads();
    }
    const float factor = s_factor[r], f = factor * cs;
#pragma unroll 1
    for (int j = j0; j < last; ++j, ++turn) {
      if (j + 1 < last) next(j + 1, turn + 1);
      if (ok) ok = mbar_wait(&bar[turn & 1], (turn >> 1) & 1);
      ap_fence_after();
      const uint32_t at = from + (turn & 1) * AW_TILE;
      const float* scales = s_scale[turn & 3] + col0;
      const int lim = see - j * AW_TILE - col0;  // of the 64 columns, those that the row sees
#pragma unroll 1
      for (int half = 0; half < 2 && 32 * (warp & 3) < rows.count; ++half) {
        float v[32];
        ap_ld32(at + 32 * half, v);
        ap_wait_ld<32>(v);
        if constexpr (S::CODES) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 k = *reinterpret_cast<const float4*>(scales + 32 * half + i);
            v[i] *= k.x, v[i + 1] *= k.y, v[i + 2] *= k.z, v[i + 3] *= k.w;
          }
        }
        if (__any_sync(0xffffffffu, lim < 32 * half + 32)) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (32 * half + i >= lim) v[i] = -INFINITY;
        }
        float top = ap_max3(v[0], v[1], v[2]);
#pragma unroll
        for (int i = 3; i < 31; i += 2) top = ap_max3(top, v[i], v[i + 1]);
        top = ap_max3(top, v[31], m);
        const float base = top == -INFINITY ? 0.f : top, off = -base * f;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 32; ++i) sum[i & 3] += at_exp2(__fmaf_rn(v[i], f, off));
        const float here = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        l = __fmaf_rn(l, at_exp2((m - base) * f), aw_exact(here, base, f, off));
        m = top;
      }
      ap_fence_before();
    }
    ok = __syncthreads_and(ok);
    if (!ok) {
      if (threadIdx.x == 0) atomicExch(status, SLS_ERR_TIMEOUT);
      // the last products of both barriers end, or run out of time too, before their columns are freed
      for (unsigned k = 1; k <= min(turn, 2u); ++k) mbar_wait(&bar[(turn - k) & 1], ((turn - k) >> 1) & 1);
      break;
    }
    if (warp >= 4) s_ml[r] = make_float2(m, l);
    __syncthreads();
    if (warp < 4 && r < rows.count) {
      const float2 o = s_ml[r];
      const float top = fmaxf(m, o.x), base = top == -INFINITY ? 0.f : top;
      l = l * at_exp2((m - base) * f) + o.y * at_exp2((o.x - base) * f);
      const float2 y = make_float2(top * factor, l);
      if (j0 == 0 && j1 == n) p.stat[rows.packed(a, w, r)] = y;
      // the part's first piece goes to slot 0, a later one (its last) to slot 1
      else p.ml[(int64_t)(2 * blockIdx.x + (t > t0)) * AW_TILE + r] = y;
    }
    __syncthreads();
    t += j1 - j0;
  }
  aw_free<2 * AW_TILE>(tmem);
}

// A warp for each row: its pieces in order.
__global__ void __launch_bounds__(32 * AW_JOIN_WARPS)
attention_weights_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AwPlan p) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * AW_JOIN_WARPS + (threadIdx.x >> 5);
  if (id >= a.T * a.q_heads) return;
  const int64_t t = ad_div(id, a.q_heads);
  const float cs = a.scale * 1.4426950408889634f;
  at_go();
  at_wait_ahead();
  int seq = (int)t;
  if (a.cu) {
    int ended = 0;
    for (int b = lane; b < c.B; b += 32) ended += a.cu[b + 1] <= t;
    seq = __reduce_add_sync(0xffffffffu, ended);
    if (seq >= c.B || t < a.cu[seq]) return;
  }
  const int hq = (int)(id - t * a.q_heads);
  const AwHead w(a, p.group, seq, hq / p.group);
  if (t >= w.q0 + w.n) return;  // offsets that do not ascend
  const int n = ad_steps<AW_TILE>(c, seq);
  float m = -INFINITY, l = 0.f;
  if (n > 0) {
    const int64_t row = (t - w.q0) * w.group + (hq - w.h * w.group), tile = row >> 7;
    const int64_t total = p.prefix[c.B];
    const int parts = (int)min((int64_t)p.ctas, total);
    const int64_t s0 = p.prefix[seq] + (w.h * aw_row_tiles(a, p.group, seq) + tile) * n, s1 = s0 + n;
    // the part of step x is the last whose start total * g / parts is at most x
    const int g0 = (int)ad_div((s0 + 1) * parts - 1, total), g1 = (int)ad_div(s1 * parts - 1, total);
    if (g0 == g1) {
      const float2 y = p.stat[id];
      m = y.x, l = y.y;
    } else {
      for (int g = g0 + lane; g <= g1; g += 32) {
        // the item's first piece is its part's last unless the part starts with it
        const int late = g == g0 && ad_div(total * g, parts) < s0;
        const float2 y = p.ml[(int64_t)(2 * g + late) * AW_TILE + (row - tile * AW_TILE)];
        const float top = fmaxf(m, y.x), base = top == -INFINITY ? 0.f : top;
        l = l * at_exp2((m - base) * cs) + y.y * at_exp2((y.x - base) * cs);
        m = top;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
        // the same order of the two addends in both lanes
        const float x = l * at_exp2((m - base) * cs), y = l2 * at_exp2((m2 - base) * cs);
        l = (lane & o) ? y + x : x + y;
        m = top;
      }
    }
  }
  __syncwarp();
  // y 2^(score cs + x) is the weight
  if (lane == 0) {
    const float x = -m * cs;
    p.stat[id] = l == 0.f ? make_float2(-INFINITY, 0.f)
                          : make_float2(x, aw_exact(1.f / l, m, cs, x));
  }
}

// ---- second pass: sums of columns ----------------------------------------------------------
template <typename E, typename KT, int HD>
__global__ void __launch_bounds__(AW_T, 2)
attention_weights_sum_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ ScaleView sc,
                             const __grid_constant__ WeightView wv, const __grid_constant__ AwPlan p,
                             int* status) {
  using S = AwShape<E, KT, HD>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ int64_t s_pre[AW_T + 1];
  __shared__ float s_factor[2 * AW_TILE];
  __shared__ __align__(16) float2 s_row[2 * AW_TILE];  // factor and summand of a row's exponents
  __shared__ __align__(16) float s_inv[2 * AW_TILE];   // factor of its weights
  __shared__ __align__(16) int s_see[2 * AW_TILE];     // tokens that it sees
  // of two units: a thread may still read its token's when another fetches the next unit's, or has
  // added it up (a head's last unit comes without a barrier before its sums)
  __shared__ float s_scale[2][AW_TILE], s_sum[2][AW_TILE];
  __shared__ uint64_t bar[2];
  __shared__ uint32_t holder;
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float cs = a.scale * 1.4426950408889634f;
  unsigned char* rows_s = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* keys_s = rows_s + 2 * S::TILE_BYTES;

  at_wait_ahead();
  if (threadIdx.x < 2) mbar_init(&bar[threadIdx.x], 1);
  mbar_fence_init();
  // sequences without rows have nothing to add
  const auto steps = [&](int s) {
    return aw_row_tiles(a, p.group, s) == 0 ? (int64_t)0 : (int64_t)ad_steps<AW_TILE>(c, s) * c.kv_heads;
  };
  const int R = ad_prefix<AW_T>(c, s_pre, nullptr, steps);
  const int64_t total = s_pre[AW_T];
  const int64_t t0 = ad_div(total * blockIdx.x, gridDim.x), t1 = ad_div(total * (blockIdx.x + 1), gridDim.x);
  if (t0 >= t1) return;
  const uint32_t tmem = aw_alloc<2 * AW_TILE>(&holder);
  const uint32_t lead = at_elect();
  int seq;
  int64_t before;
  ad_find<AW_T>(s_pre, R, t0, steps, seq, before);
  // this thread's token of a tile, and its rows
  const int r = 32 * (warp & 3) + lane, col0 = 64 * (warp >> 2);
  const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + col0;
  unsigned phase[2] = {0, 0};
  bool ok = true, live[2];
  AwKeys<E, KT, HD> keys;
  // the unit after the next: its head, first token and pages, a unit ahead of its keys
  int n = ad_steps<AW_TILE>(c, seq), plan0;
  AwHead ahead(a, p.group, seq, (int)ad_div(t0 - before, n));
  int tile = (int)(t0 - before - (int64_t)ahead.h * n);
  auto plan = [&] {
    plan0 = tile * AW_TILE;
    keys.pages(a, ahead, plan0);
  };
  auto advance = [&] {
    if (++tile == n) {
      tile = 0;
      if (++ahead.h == c.kv_heads) {
        do ++seq;
        while (steps(seq) == 0);
        n = ad_steps<AW_TILE>(c, seq);
        ahead = AwHead(a, p.group, seq, 0);
      }
    }
    plan();
  };
  // two tiles of rows (or one) to shared memory
  auto stage = [&](const AwHead& w, const AwRows& r0, const AwRows& r1) {
    aw_stage_rows<E, KT, HD>(a, w, r0, rows_s, s_factor);
    if (r1.count > 0) aw_stage_rows<E, KT, HD>(a, w, r1, rows_s + S::TILE_BYTES, s_factor + AW_TILE);
    const int k = threadIdx.x & (AW_TILE - 1);
    const AwRows& mine = threadIdx.x < AW_TILE ? r0 : r1;
    float2 stat = make_float2(-INFINITY, 0.f);
    if (k < mine.count) stat = p.stat[mine.packed(a, w, k)];
    __syncthreads();
    s_row[threadIdx.x] = make_float2(s_factor[threadIdx.x] * cs, stat.x);
    s_inv[threadIdx.x] = stat.y;
    s_see[threadIdx.x] = mine.see(a, w, k);
  };
  // products of a tile; one whose last row sees none of the tokens adds nothing
  auto issue = [&](int i, const AwHead& w, const AwRows& rows, int start) {
    live[i] = rows.count > 0 && rows.see(a, w, rows.count - 1) > start;
    if (live[i] && warp == 0) {
      ap_fence_after();
      aw_products<E, KT, HD>(lead, tmem + i * AW_TILE, keys_s, rows_s + i * S::TILE_BYTES, &bar[i]);
    }
  };
  auto wait = [&](int i) {
    if (!live[i]) return;
    if (ok) ok = mbar_wait(&bar[i], phase[i]);
    phase[i] ^= 1;
    ap_fence_after();
  };
  float col[4];
  auto add = [&](int i, int count, int start, float scale) {
    const int row0 = i * AW_TILE + col0, x = start + r;
    // rows in order see ever more: the first of the 64 sees all of these tokens, or not
    const bool whole = col0 + 63 < count && s_see[row0] >= start + AW_TILE;
#pragma unroll 1
    for (int half = 0; half < 64 && col0 + half < count; half += 32) {
      float v[32];
      ap_ld32(from + i * AW_TILE + half, v);
      ap_wait_ld<32>(v);
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 f = *reinterpret_cast<const float4*>(&s_row[row0 + half + k]);
        const float4 g = *reinterpret_cast<const float4*>(&s_row[row0 + half + k + 2]);
        if constexpr (S::CODES) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[k + j] *= scale;
        }
        const float4 y = *reinterpret_cast<const float4*>(&s_inv[row0 + half + k]);
        const float by[4] = {y.x, y.y, y.z, y.w};
        const float e[4] = {at_exp2(__fmaf_rn(v[k], f.x, f.y)), at_exp2(__fmaf_rn(v[k + 1], f.z, f.w)),
                            at_exp2(__fmaf_rn(v[k + 2], g.x, g.y)),
                            at_exp2(__fmaf_rn(v[k + 3], g.z, g.w))};
        if (whole) {
#pragma unroll
          for (int j = 0; j < 4; ++j) col[j] = __fmaf_rn(e[j], by[j], col[j]);
        } else {
          const int4 see = *reinterpret_cast<const int4*>(&s_see[row0 + half + k]);
          const int s[4] = {see.x, see.y, see.z, see.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (x < s[j]) col[j] = __fmaf_rn(e[j], by[j], col[j]);
        }
      }
    }
    ap_fence_before();
  };

  // The first two tiles of rows of a head stay in shared memory from unit to unit, and the products
  // of a unit's first tile run while the scores of the last unit's second are worked on.
  plan();
  AwHead next = ahead;
  int key0 = plan0;
  keys.load(a, sc, next, key0);
  if (t0 + 1 < t1) advance();
  AwRows r0(next, 0), r1(next, 1);
  bool begin = true;
  float scale = 1.f;
#pragma unroll 1
  for (int64_t t = t0; t < t1; ++t) {
    const AwHead w = next;
    const int start = key0, x = start + r;
    const int64_t tiles = (w.rows + AW_TILE - 1) >> 7;
    if (begin) {
      r0 = AwRows(w, 0), r1 = AwRows(w, 1);
      stage(w, r0, r1);
      keys.store(keys_s, s_scale[t & 1]);
      aw_fence();
      __syncthreads();
      issue(0, w, r0, start);
      issue(1, w, r1, start);
      if constexpr (S::CODES) scale = s_scale[t & 1][r];
    }
    const float mine = scale;
    // the token's weight so far, and the next unit's keys
    float* to = nullptr;
    float was = 0.f;
    if (warp < 4 && x < w.len) {
      const int64_t page = c.table[w.seq * c.table_ld + (x >> c.page_shift)];
      if (page >= 0 && page < c.num_pages) {
        to = wv.data + page * wv.page + w.h * wv.head + (x & ((1 << c.page_shift) - 1));
        was = *to;
      }
    }
    if (t + 1 < t1) {
      next = ahead;
      key0 = plan0;
      keys.load(a, sc, next, key0);
      if (t + 2 < t1) advance();
    }
    const bool same = t + 1 < t1 && next.seq == w.seq && next.h == w.h && tiles <= 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) col[j] = 0.f;
    wait(0);
    if (live[0]) add(0, r0.count, start, mine);
    wait(1);
    const bool second = live[1];
    if (same) {
      // the unit's products are done: its keys' place is free; at the barrier so are the first
      // tile's columns
      keys.store(keys_s, s_scale[(t + 1) & 1]);
      aw_fence();
      __syncthreads();
      issue(0, w, r0, key0);
      if constexpr (S::CODES) scale = s_scale[(t + 1) & 1][r];
    }
    if (second) add(1, r1.count, start, mine);
#pragma unroll 1
    for (int64_t b = 2; b < tiles; b += 2) {
      const AwRows a0(w, b), a1(w, b + 1);
      __syncthreads();
      stage(w, a0, a1);
      aw_fence();
      __syncthreads();
      issue(0, w, a0, start);
      issue(1, w, a1, start);
      wait(0);
      if (live[0]) add(0, a0.count, start, mine);
      wait(1);
      if (live[1]) add(1, a1.count, start, mine);
    }
    const float sum = (col[0] + col[1]) + (col[2] + col[3]);
    if (warp >= 4) s_sum[t & 1][r] = sum;
    // and the second tile's columns are read
    ok = __syncthreads_and(ok);
    if (!ok) {
      if (threadIdx.x == 0) atomicExch(status, SLS_ERR_TIMEOUT);
      // as in the first pass; the next unit's first products are issued where it is the same head's
      for (int i = 0; i < 2; ++i) mbar_wait(&bar[i], phase[i] ^ 1);
      if (same && live[0]) mbar_wait(&bar[0], phase[0]);
      break;
    }
    if (same) issue(1, w, r1, key0);
    begin = !same;
    if (to) *to = was + (sum + s_sum[t & 1][r]);
  }
  aw_free<2 * AW_TILE>(tmem);
}

struct AwHost {
  int ctas;
  size_t prefix_b, ml_b, stat_b;
};

int aw_host(const CacheView& c, int64_t T, int q_heads, AwHost* h) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  h->ctas = 2 * sms;
  h->prefix_b = sls_align256(((size_t)c.B + 1) * 8);
  h->ml_b = sls_align256((size_t)h->ctas * 2 * AW_TILE * 8);
  h->stat_b = sls_align256((size_t)T * q_heads * 8);
  return SLS_OK;
}

template <typename E, typename KT, int HD>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, const AwHost& h,
           void* workspace, cudaStream_t stream) {
  using S = AwShape<E, KT, HD>;
  static bool set[64] = {};  // per device
  static int* words[64] = {};
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  constexpr size_t smem1 = 3 * S::TILE_BYTES + 1024, smem2 = 3 * S::TILE_BYTES + 1024;
  auto first = attention_weights_rows_kernel<E, KT, HD>;
  auto second = attention_weights_sum_kernel<E, KT, HD>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(first, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem1));
    SLS_CUDA_TRY(
        cudaFuncSetAttribute(second, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem2));
  }
  int* word = dev < 64 ? words[dev] : nullptr;
  if (!word) {
    const int st = decode_status_word(&word);
    if (st != SLS_OK) return st;
  }
  if (dev < 64) words[dev] = word, set[dev] = true;
  AwPlan p;
  char* at = (char*)workspace;
  p.group = a.q_heads / a.c.kv_heads;
  p.ctas = h.ctas;
  p.prefix = (int64_t*)at;
  p.ml = (float2*)(at += h.prefix_b);
  p.stat = (float2*)(at + h.ml_b);
  int st = at_launch(first, dim3((unsigned)h.ctas), AW_T, smem1, 1, stream, a, s, p, word);
  if (st != SLS_OK) return st;
  const int64_t all = a.T * a.q_heads;
  st = at_launch(attention_weights_join_kernel,
                 dim3((unsigned)((all + AW_JOIN_WARPS - 1) / AW_JOIN_WARPS)), 32 * AW_JOIN_WARPS, 0, 1,
                 stream, a, p);
  if (st != SLS_OK) return st;
  return at_launch(second, dim3((unsigned)h.ctas), AW_T, smem2, 1, stream, a, s, w, p, word);
}

template <typename E, typename KT>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, const AwHost& h,
           void* workspace, cudaStream_t stream) {
  return a.c.head_dim > 64 ? launch<E, KT, 128>(a, s, w, h, workspace, stream)
                           : launch<E, KT, 64>(a, s, w, h, workspace, stream);
}

template <typename E>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code, const AwHost& h,
           void* workspace, cudaStream_t stream) {
  return code == SLS_I8     ? launch<E, I8>(a, s, w, h, workspace, stream)
         : code == SLS_E4M3 ? launch<E, E4M3>(a, s, w, h, workspace, stream)
                            : launch<E, E>(a, s, w, h, workspace, stream);
}

}  // namespace

size_t attention_weights_workspace(const CacheView& c, int64_t T, int q_heads) {
  if (c.B == 0 || T == 0 || c.max_pages == 0) return 0;
  if (attention_weights_few(c, T, q_heads))
    return attention_weights_few_workspace(c, T, q_heads);
  AwHost h;
  return aw_host(c, T, q_heads, &h) == SLS_OK ? h.prefix_b + h.ml_b + h.stat_b : 0;
}

int launch_attention_weights(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code,
                             int dtype, void* workspace, cudaStream_t stream) {
  if (a.c.B == 0 || a.T == 0 || a.c.max_pages == 0) return SLS_OK;
  if (a.T * a.q_heads > (int64_t)0x7fffffff * AW_JOIN_WARPS) return SLS_ERR_UNSUPPORTED;
  if (attention_weights_few(a.c, a.T, a.q_heads))
    return launch_attention_weights_few(a, s, w, code, dtype, workspace, stream);
  AwHost h;
  const int st = aw_host(a.c, a.T, a.q_heads, &h);
  if (st != SLS_OK) return st;
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, s, w, code, h, workspace, stream)
                           : launch<__half>(a, s, w, code, h, workspace, stream);
}

}  // namespace sls
