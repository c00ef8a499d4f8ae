// Accumulated attention weights where a sequence has few rows (a decode step: one token): keys
// are read once, as the decode kernels read them, and the scores kept.
//
// Bound by HBM bandwidth.  The first launch is decode without values: a warp owns a key head of a
// part of all sequences' steps of 32 tokens, keys are the 16-row operands and rows (token, query
// head) the 8 columns, and scores go to the workspace, 4 bytes a row and token (four rows': a
// sixteenth of a 16-bit key of 128 elements; places for as many tokens as the page table holds), with
// maximum and sum of every piece.  A sequence of
// more rows is gone through again for each AF_ROWS of them.  The second launch has a thread for each
// token: it joins the pieces of every row in order and adds up the row's weights.  32 sequences to
// 4096 tokens, 32 + 8 heads of 128, bfloat16: 39.4 us, 3.9 TB/s of keys (31 us for the scores, in
// parts of some 18 steps a warp; the sum's launch overlaps their end).
#include <algorithm>

#include "attention_decode.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int AF_SUM_T = 256;
constexpr int AF_UNIT = 4 * AF_SUM_T;  // tokens of a CTA of the second launch
constexpr int AF_AHEAD = 4;            // rows whose scores it fetches first
constexpr int64_t AF_MOST_SCORES = (int64_t)1 << 28;

// SIZE: bytes of an element of keys
template <int HD, int SIZE>
struct AfShape {
  static constexpr int WARPS = 12;
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int ROW = HD * SIZE < 128 ? HD * SIZE : 128;  // bytes of a row of a copy
  static constexpr int HALVES = HD * SIZE / ROW;
  static constexpr int HALF_BYTES = AD_KEYS * ROW;
  static constexpr int STAGE_BYTES = HALVES * HALF_BYTES;
  static constexpr int STAGES = 16384 / STAGE_BYTES;
  static constexpr int READS = HD * SIZE / 64;  // 16-byte reads of a key for each of four lanes
  static constexpr size_t SMEM = (size_t)WARPS * STAGES * STAGE_BYTES + 1024;
  // Byte of 16-byte chunk ch of a key, as the copies' swizzle left it.
  SLS_DEV static int at(int key, int ch) {
    if constexpr (ROW == 128) return (ch >> 3) * HALF_BYTES + key * 128 + (((ch & 7) ^ (key & 7)) << 4);
    else return key * 64 + ((ch ^ (key >> 1 & 3)) << 4);
  }
};

constexpr int AF_ROWS = 8;  // of a pass

struct AfPlan {
  int groups;        // most parts
  int64_t* prefix;   // B + 1: steps of all passes before every sequence
  float2* ml;        // (part, first or last piece, key head, row): maximum of the scores, sum
  float2* stat;      // (token, query head): the same of a pass that one part has whole
  float* scores;     // (token, query head, cache index)
  int64_t room;
};

// Packed rows of a sequence.
SLS_DEV void af_tokens(const AttnArgs& a, int seq, int64_t& q0, int64_t& q1) {
  if (a.cu) seq_rows(a.cu, seq, a.T, q0, q1);
  else q0 = seq, q1 = seq + 1;
}

SLS_DEV int af_passes(const AttnArgs& a, int seq) {
  int64_t q0, q1;
  af_tokens(a, seq, q0, q1);
  return (int)(((q1 - q0) * (a.q_heads / a.c.kv_heads) + AF_ROWS - 1) / AF_ROWS);
}

template <typename E, typename KT, int HD>
__global__ void __launch_bounds__(AfShape<HD, sizeof(KT) == 2 ? 2 : 1>::THREADS, 1)
attention_scores_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ AttnArgs a,
                        const __grid_constant__ ScaleView sc, const __grid_constant__ AfPlan p,
                        int* status) {
  constexpr bool CODES = !std::is_same<E, KT>::value;
  using S = AfShape<HD, CODES ? 1 : 2>;
  using M = typename std::conditional<CODES, __half, E>::type;
  constexpr int AD_T = S::THREADS, KS = HD / 16;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ int64_t s_pre[AD_T + 1];
  __shared__ float2 s_scale[S::WARPS][S::STAGES];
  __shared__ uint64_t full_bar[S::WARPS][S::STAGES];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, cq = lane & 3;
  const int group = a.q_heads / c.kv_heads;
  const float cs = a.scale * 1.4426950408889634f;

  at_wait_ahead();
  if (lane < S::STAGES) mbar_init(&full_bar[warp][lane], 1);
  mbar_fence_init();
  const auto steps = [&](int s) { return (int64_t)ad_steps(c, s) * af_passes(a, s); };
  const int R = ad_prefix<AD_T>(c, s_pre, p.prefix, steps);
  const int64_t total = s_pre[AD_T];
  const int parts = ad_parts(total, p.groups);
  const int gw = blockIdx.x * S::WARPS + warp;
  const int g = gw / c.kv_heads, kvh = gw - g * c.kv_heads;
  if (g >= parts) return;
  const int64_t t0 = ad_div(total * g, parts), t1 = ad_div(total * (g + 1), parts);
  int seq;
  int64_t before;  // steps before seq
  ad_find<AD_T>(s_pre, R, t0, steps, seq, before);

  unsigned char* ring = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023) +
                        warp * S::STAGES * S::STAGE_BYTES;
  uint64_t* bars = full_bar[warp];
  float2* scales = s_scale[warp];
  const uint32_t lead = at_elect();
  // ---- copies ahead: the step to issue next, as in the decode kernels
  int is = seq, ilen = (int)cache_len(c, seq), isteps = ad_steps(c, seq);
  int64_t ileft = steps(seq) - (t0 - before);  // steps of this sequence, all passes, to issue
  int ij = (int)(t0 - before - ad_div(t0 - before, isteps) * isteps);
  int64_t left = t1 - t0;
  int batch0 = -1, page = -1;
  unsigned issued = 0, used = 0;
  auto issue = [&] {
    if (left > 0) {
      if (ij == isteps) ij = 0, batch0 = -1;
      if (ileft == 0) {
        do ++is;
        while ((ileft = steps(is)) == 0);
        ilen = (int)cache_len(c, is);
        isteps = ad_steps(c, is);
        ij = 0;
        batch0 = -1;
      }
      if (batch0 < 0 || ij - batch0 == 16) {
        batch0 = ij;
        const int x = ij * AD_KEYS + 16 * lane;
        page = x < ilen ? c.table[is * c.table_ld + (x >> c.page_shift)] : -1;
      }
      const unsigned st = issued % S::STAGES;
      const int box = min(AD_KEYS, 1 << c.page_shift);
      const int copies = (min(AD_KEYS, ilen - ij * AD_KEYS) + box - 1) / box;
      const int slot0 = (ij * AD_KEYS) & ((1 << c.page_shift) - 1);
      if (lead) mbar_expect_tx(&bars[st], S::HALVES * copies * box * S::ROW);
      __syncwarp();
      const int first = 2 * (ij - batch0);
#pragma unroll 1
      for (int cp = 0; cp < copies; ++cp) {
        const int pg = __shfl_sync(0xffffffffu, page, first + cp);
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h)
          at_tma4(lead, smem_u32(ring) + st * S::STAGE_BYTES + h * S::HALF_BYTES + cp * box * S::ROW,
                  &tmK, 64 * h, slot0, kvh, pg, &bars[st]);
      }
      if constexpr (CODES) {
        const int half = lane & 1;
        const int64_t pg = __shfl_sync(0xffffffffu, page, first + half);
        if (lane < 2) {
          const int slot = (ij * AD_KEYS + 16 * half) & ((1 << c.page_shift) - 1);
          const bool real = ij * AD_KEYS + 16 * half < ilen && pg >= 0 && pg < c.num_pages;
          const float* f = sc.k;
          if (real) f += pg * sc.page + (slot >> sc.shift) * sc.block + kvh * sc.head;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(
                           smem_u32(scales + st) + 4 * lane),
                       "l"(f), "r"(real ? 4 : 0)
                       : "memory");
        }
      }
      ++ij;
      ++issued;
      --ileft;
      --left;
    }
    if constexpr (CODES) asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < S::STAGES; ++i) issue();

  int64_t t = t0;
  while (t < t1) {
    // ---- a piece: steps [j0, j1) of a pass over sequence seq ----
    const int len = (int)cache_len(c, seq), n = ad_steps(c, seq);
    const int64_t all = steps(seq);
    if (all == 0) {
      ++seq;
      continue;
    }
    const int pass = (int)ad_div(t - before, n);
    const int j0 = (int)((t - before) - (int64_t)pass * n);
    const int j1 = (int)min((int64_t)n, j0 + t1 - t);
    int64_t q0, q1;
    af_tokens(a, seq, q0, q1);
    const int rows = (int)((q1 - q0) * group), row0 = pass * AF_ROWS;
    // this lane's operand row, and the two of its columns
    uint32_t q[KS][2];
    float qf[2];
    {
      const int row = row0 + r, tok = row / group;
      const char* qp = a.q.data + (q0 + tok) * a.q.token_b + (kvh * group + row - tok * group) * a.q.head_b;
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int e = CODES ? 64 * (k >> 2) + 16 * cq + 4 * (k & 3) : 32 * (k >> 1) + 8 * cq + 4 * (k & 1);
        uint2 raw = make_uint2(0u, 0u);
        if (row < rows && e < c.head_dim) raw = *reinterpret_cast<const uint2*>(qp + 2 * e);
        const float2 f = Half2<E>::widen(raw.x), h = Half2<E>::widen(raw.y);
        top = fmaxf(fmaxf(fmaxf(top, fabsf(f.x)), fmaxf(fabsf(f.y), fabsf(h.x))), fabsf(h.y));
        q[k][0] = raw.x, q[k][1] = raw.y;
      }
      float back = 1.f;
      if constexpr (!std::is_same<E, M>::value) {
        // bfloat16 to float16: the largest element to [2^14, 2^15)
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = max(__float_as_int(top) >> 23, 16);
        const float by = __int_as_float((127 + 14 + 127 - e) << 23);
        back = __int_as_float((e - 14) << 23);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 f = Half2<E>::widen(q[k][i]);
            q[k][i] = Half2<__half>::narrow(f.x * by, f.y * by);
          }
      }
      qf[0] = __shfl_sync(0xffffffffu, back, 8 * cq);
      qf[1] = __shfl_sync(0xffffffffu, back, 8 * cq + 4);
    }
    float* out[2];
    int see[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + 2 * cq + i, tok = row / group;
      out[i] = row < rows ? p.scores + ((q0 + tok) * a.q_heads + kvh * group + row - tok * group) * p.room
                          : nullptr;
      see[i] = row >= rows ? len : a.causal ? len - (int)(q1 - q0) + tok + 1 : len;
    }
    const int least = min(__reduce_min_sync(0xffffffffu, see[0]), __reduce_min_sync(0xffffffffu, see[1]));
    float mx[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
      if constexpr (CODES) asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
      const unsigned st = used % S::STAGES;
      if (!__all_sync(0xffffffffu, mbar_wait(&bars[st], (used / S::STAGES) & 1))) {
        if (lane == 0) atomicExch(status, SLS_ERR_TIMEOUT);
        for (unsigned x = used + 1; x < issued; ++x)
          mbar_wait(&bars[x % S::STAGES], (x / S::STAGES) & 1);
        return;
      }
      __syncwarp();  // the scales are copied by lanes 0 and 1
      const unsigned char* stage = ring + st * S::STAGE_BYTES;
      float s[2][4];
      const int mine = ad_token(r);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        s[mt][0] = s[mt][1] = s[mt][2] = s[mt][3] = 0.f;
#pragma unroll
        for (int i = 0; i < S::READS; ++i) {
          const uint4 u = *reinterpret_cast<const uint4*>(stage + S::at(16 * mt + mine, 4 * i + cq));
          const uint4 v = *reinterpret_cast<const uint4*>(stage + S::at(16 * mt + mine + 8, 4 * i + cq));
          const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v.x, v.y, v.z, v.w};
          if constexpr (CODES) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              uint32_t k[4];
              codes_half<KT>(uw[y], k[0], k[2]);
              codes_half<KT>(vw[y], k[1], k[3]);
              mma16816<M>(s[mt], k, q[4 * i + y][0], q[4 * i + y][1]);
            }
          } else {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t k[4] = {uw[2 * y], vw[2 * y], uw[2 * y + 1], vw[2 * y + 1]};
              mma16816<M>(s[mt], k, q[2 * i + y][0], q[2 * i + y][1]);
            }
          }
        }
      }
      if constexpr (CODES) {
        const float2 f = scales[st];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0][i] *= f.x * qf[i & 1], s[1][i] *= f.y * qf[i & 1];
      }
      const int x0 = j * AD_KEYS;
      if (x0 + AD_KEYS > least) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (x0 + 16 * mt + mine + 8 * (i >> 1) >= see[i & 1]) s[mt][i] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (out[i]) {
          float* to = out[i] + x0 + mine;
          to[0] = s[0][i], to[8] = s[0][2 + i], to[16] = s[1][i], to[24] = s[1][2 + i];
        }
        // maxima and sums of this lane's own tokens: joined at the end of the piece
        const float m = fmaxf(fmaxf(fmaxf(s[0][i], s[0][2 + i]), fmaxf(s[1][i], s[1][2 + i])), mx[i]);
        const float base = m == -INFINITY ? 0.f : m;
        l[i] = l[i] * at_exp2((mx[i] - base) * cs) +
               ((at_exp2((s[0][i] - base) * cs) + at_exp2((s[0][2 + i] - base) * cs)) +
                (at_exp2((s[1][i] - base) * cs) + at_exp2((s[1][2 + i] - base) * cs)));
        mx[i] = m;
      }
      __syncwarp();
      ++used;
      issue();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float m = mx[i];
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      const float base = m == -INFINITY ? 0.f : m;
      float x = l[i] * at_exp2((mx[i] - base) * cs);
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      const int row = row0 + 2 * cq + i, tok = row / group;
      if (r != 0 || row >= rows) continue;
      if (j0 == 0 && j1 == n)
        p.stat[(q0 + tok) * a.q_heads + kvh * group + row - tok * group] = make_float2(m, x);
      else
        // the part's first piece goes to slot 0, a later one (its last) to slot 1
        p.ml[((int64_t)(2 * g + (t > t0)) * c.kv_heads + kvh) * AF_ROWS + 2 * cq + i] =
            make_float2(m, x);
    }
    t += j1 - j0;
    if (t == before + all) {
      before += all;
      ++seq;
    }
  }
}

// A CTA for each 1024 tokens of a sequence and key head, a thread for four.
__global__ void __launch_bounds__(AF_SUM_T)
attention_scores_sum_kernel(const __grid_constant__ AttnArgs a,
                            const __grid_constant__ WeightView wv, const __grid_constant__ AfPlan p) {
  __shared__ float2 s_stat[AF_SUM_T];
  const CacheView& c = a.c;
  const int group = a.q_heads / c.kv_heads;
  const float cs = a.scale * 1.4426950408889634f;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.y;
  at_go();
  at_wait_ahead();
  const int units = (int)(p.room / AF_UNIT);
  const int seq = blockIdx.x / units;
  const int x0 = (blockIdx.x - seq * units) * AF_UNIT, x = x0 + 4 * threadIdx.x;
  const int len = (int)cache_len(c, seq);
  if (x0 >= len) return;
  int64_t q0, q1;
  af_tokens(a, seq, q0, q1);
  const int64_t rows = (q1 - q0) * group;
  const int64_t total = p.prefix[c.B], first = p.prefix[seq];
  const int parts = ad_parts(total, p.groups);
  const int n = ad_steps(c, seq);
  // the first rows' scores and the tokens' weights so far are fetched while the pieces are joined
  const float* sp = p.scores + (q0 * a.q_heads + h * group) * p.room + x;
  auto scores = [&](int64_t row) {
    const int64_t tok = ad_div(row, group);
    return *reinterpret_cast<const float4*>(sp + (tok * a.q_heads + (row - tok * group)) * p.room);
  };
  float4 ahead[AF_AHEAD];
#pragma unroll
  for (int i = 0; i < AF_AHEAD; ++i)
    if (x < len && i < rows) ahead[i] = scores(i);
  float4 was = make_float4(0.f, 0.f, 0.f, 0.f);
  float* to = nullptr;  // four slots of one page
  if (x < len && rows > 0) {
    const int64_t page = c.table[seq * c.table_ld + (x >> c.page_shift)];
    if (page >= 0 && page < c.num_pages) {
      to = wv.data + page * wv.page + h * wv.head + (x & ((1 << c.page_shift) - 1));
      was = *reinterpret_cast<const float4*>(to);
    }
  }
  float w[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t b0 = 0; b0 < rows; b0 += AF_SUM_T) {
    const int here = (int)min((int64_t)AF_SUM_T, rows - b0);
    __syncthreads();
    for (int i = warp; i < here; i += AF_SUM_T / 32) {
      const int64_t row = b0 + i, tok = ad_div(row, group);
      const int64_t pass = row / AF_ROWS;
      const int64_t s0 = first + pass * n, s1 = s0 + n;  // steps of the row's pass
      // the part of step t is the last whose start total * g / parts is at most t
      const int g0 = (int)ad_div((s0 + 1) * parts - 1, total), g1 = (int)ad_div(s1 * parts - 1, total);
      float m = -INFINITY, l = 0.f;
      if (g0 == g1) {
        const float2 y = p.stat[(q0 + tok) * a.q_heads + h * group + (row - tok * group)];
        m = y.x, l = y.y;
      } else {
        for (int g = g0 + lane; g <= g1; g += 32) {
          // the pass's first piece is its part's last unless the part starts with it
          const int late = g == g0 && ad_div(total * g, parts) < s0;
          const float2 y =
              p.ml[((int64_t)(2 * g + late) * c.kv_heads + h) * AF_ROWS + (row - pass * AF_ROWS)];
          const float top = fmaxf(m, y.x), base = top == -INFINITY ? 0.f : top;
          l = l * at_exp2((m - base) * cs) + y.y * at_exp2((y.x - base) * cs);
          m = top;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
          const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
          // the same order of the two addends in both lanes
          const float u = l * at_exp2((m - base) * cs), v = l2 * at_exp2((m2 - base) * cs);
          l = (lane & o) ? v + u : u + v;
          m = top;
        }
      }
      if (lane == 0) s_stat[i] = make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
    auto add = [&](const float4& f, int i) {
      const float s[4] = {f.x, f.y, f.z, f.w};
      const float2 y = s_stat[i];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] += s[k] == -INFINITY ? 0.f : at_exp2((s[k] - y.x) * cs) * y.y;
    };
    if (x < len) {
      if (b0 == 0)
#pragma unroll
        for (int i = 0; i < AF_AHEAD; ++i)
          if (i < here) add(ahead[i], i);
      for (int i = b0 == 0 ? AF_AHEAD : 0; i < here; ++i) add(scores(b0 + i), i);
    }
  }
  if (!to) return;
  // those past the end are left as they are
  if (x + 4 <= len)
    *reinterpret_cast<float4*>(to) =
        make_float4(was.x + w[0], was.y + w[1], was.z + w[2], was.w + w[3]);
  else
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (x + k < len) to[k] += w[k];
}

struct AfHost {
  int groups, grid;
  int64_t room;
  size_t prefix_b, ml_b, stat_b, score_b;
};

int af_host(const CacheView& c, int64_t T, int q_heads, AfHost* h) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  constexpr int warps = AfShape<128, 2>::WARPS;
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const int64_t rows = T * (q_heads / c.kv_heads);
  h->room = (cap + AF_UNIT - 1) / AF_UNIT * AF_UNIT;
  // no more parts than there can be steps in: every sequence's rows but AF_ROWS - 1 fill passes
  const int64_t most = (rows / AF_ROWS + c.B) * (cap / AD_KEYS + 1);
  h->groups = (int)std::min<int64_t>(std::max(1, sms * warps / c.kv_heads),
                                     (most + AD_MIN_STEPS - 1) / AD_MIN_STEPS);
  h->grid = (h->groups * c.kv_heads + warps - 1) / warps;
  h->prefix_b = sls_align256(((size_t)c.B + 1) * 8);
  h->ml_b = sls_align256((size_t)h->groups * 2 * c.kv_heads * AF_ROWS * 8);
  h->stat_b = sls_align256((size_t)T * q_heads * 8);
  h->score_b = sls_align256((size_t)T * q_heads * h->room * 4);
  return SLS_OK;
}

template <typename E, typename KT, int HD>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, const AfHost& h,
           void* workspace, cudaStream_t stream) {
  constexpr int SIZE = std::is_same<E, KT>::value ? 2 : 1;
  using S = AfShape<HD, SIZE>;
  static bool set[64] = {};  // per device
  static int* words[64] = {};
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto kern = attention_scores_kernel<E, KT, HD>;
  if (dev >= 64 || !set[dev])
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::SMEM));
  int* word = dev < 64 ? words[dev] : nullptr;
  if (!word) {
    const int st = decode_status_word(&word);
    if (st != SLS_OK) return st;
  }
  if (dev < 64) words[dev] = word, set[dev] = true;
  const CacheView& c = a.c;
  CUtensorMap map;
  const int slots = std::min(AD_KEYS, 1 << c.page_shift);
  if (SIZE == 2 ? !at_cache_map(&map, std::is_same<E, __half>::value ? SLS_F16 : SLS_BF16, c, c.k, slots)
                : !at_code_map<HD>(&map, c, c.k, slots))
    return SLS_ERR_UNSUPPORTED;
  AfPlan p;
  char* at = (char*)workspace;
  p.groups = h.groups;
  p.room = h.room;
  p.prefix = (int64_t*)at;
  p.ml = (float2*)(at += h.prefix_b);
  p.stat = (float2*)(at += h.ml_b);
  p.scores = (float*)(at + h.stat_b);
  const int st = at_launch(kern, dim3((unsigned)h.grid), S::THREADS, S::SMEM, 1, stream, map, a, s,
                           p, word);
  if (st != SLS_OK) return st;
  return at_launch(attention_scores_sum_kernel,
                   dim3((unsigned)(c.B * (h.room / AF_UNIT)), (unsigned)c.kv_heads), AF_SUM_T, 0, 1,
                   stream, a, w, p);
}

template <typename E, typename KT>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, const AfHost& h,
           void* workspace, cudaStream_t stream) {
  return a.c.head_dim > 64 ? launch<E, KT, 128>(a, s, w, h, workspace, stream)
                           : launch<E, KT, 64>(a, s, w, h, workspace, stream);
}

template <typename E>
int launch(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code, const AfHost& h,
           void* workspace, cudaStream_t stream) {
  return code == SLS_I8     ? launch<E, I8>(a, s, w, h, workspace, stream)
         : code == SLS_E4M3 ? launch<E, E4M3>(a, s, w, h, workspace, stream)
                            : launch<E, E>(a, s, w, h, workspace, stream);
}

}  // namespace

// Up to 32 rows a sequence on average.  8 sequences to 8192 tokens, 8 key heads of 128, 4 / 8 / 16 /
// 32 / 64 rows: bfloat16 keys 19 / 22 / 30 / 47 / 87 us here, 60 / 60 / 61 / 60 / 64 in two passes;
// e4m3 15 / 19 / 27 / 45 / 80 and 52 / 52 / 53 / 50 / 55.  The average does for ragged rows too: 400
// tokens of 32 + 8 heads in one sequence beside 63 single ones, 4096 cached each, 1316 us here (200
// times through the one's keys), 2175 in two passes.
//
// Scores have places for all that the page table can hold, so that their room is what a wide table
// costs: up to 1 GiB of them.  256 single tokens of 32 heads over up to 2048, a table of 131072: 359 us
// here with 4 GiB, 558 in two passes without.
bool attention_weights_few(const CacheView& c, int64_t T, int q_heads) {
  const int64_t room = (((int64_t)c.max_pages << c.page_shift) + AF_UNIT - 1) / AF_UNIT;
  return T * (q_heads / c.kv_heads) <= 32 * (int64_t)c.B && c.B * room <= 0x7fffffff &&
         c.kv_heads <= 65535 && T * q_heads <= AF_MOST_SCORES / (room * AF_UNIT);
}

size_t attention_weights_few_workspace(const CacheView& c, int64_t T, int q_heads) {
  AfHost h;
  if (af_host(c, T, q_heads, &h) != SLS_OK) return 0;
  return h.prefix_b + h.ml_b + h.stat_b + h.score_b;
}

int launch_attention_weights_few(const AttnArgs& a, const ScaleView& s, const WeightView& w,
                                 int code, int dtype, void* workspace, cudaStream_t stream) {
  AfHost h;
  const int st = af_host(a.c, a.T, a.q_heads, &h);
  if (st != SLS_OK) return st;
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, s, w, code, h, workspace, stream)
                           : launch<__half>(a, s, w, code, h, workspace, stream);
}

}  // namespace sls
