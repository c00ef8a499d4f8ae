// New keys (normalised, rotated) and values as 8-bit codes: a power-of-two scale for each block
// of a page's slots and key head,
//   s' = max(|s|, 2^e), 2^e the least with max|y| <= Q 2^e,   c = round(y / s'),
// s the scale of a block that holds earlier tokens, whose codes c become round(c s / s') where that
// is not s.
//
// A CTA takes blocks whose first new token lies among its `tile` packed tokens, one after the
// other, and all or a share of their heads: cosines and sines are formed once for all heads.
// A lane holds sixteen elements of a token's head, four or eight lanes a row.  A warp has a head of
// a block to itself and goes over its rows twice, the second time from the caches: rows kept in
// registers between the maximum and the codes need all of a CTA's warps for one head, and a barrier
// for each.
//
// The queries go through the 16-bit append's kernel, with no key heads, which starts while the last
// CTAs here run (21345 tokens: 131 us one after the other); those of few tokens are turned by CTAs of
// this launch.
//
// Bound by memory in the limit; keys and values are held up by latency and instructions instead (16
// warps an SM, 41% of issue slots, 20% of DRAM's rate in a profile of them alone), which the queries'
// launch makes up for in part.  21345 tokens of 32 + 8 heads of 128, e4m3: 113.9 us, 4.2 TB/s; 10717
// tokens of 25 + 5 heads of 64, int8: 18.6 us, 2.9 TB/s; 4 single tokens 3.9 us, latency.  In a trace
// of the first a CTA of keys forms its factors in 9000 cycles and goes over its rows in 31000 and
// 15000, one of values in 16000 and 9000.
#include <algorithm>

#include "attention_turn.cuh"
#include "cache8.cuh"

namespace sls {

namespace {

constexpr int Q8_T = 256;
// rows as they come; halves of whole vectors; pairs side by side; halves that split vectors
enum { Q8_PLAIN, Q8_HALVES, Q8_SIDES, Q8_ODD };
constexpr int Q8_WARPS = 1216, Q8_CTAS = 912;  // at least so many, heads permitting: for 152 SMs
// New tokens of a block up to which a head is one group's (64 sequences of 2 / 3 / 4 / 6 / 8 tokens,
// 4 heads of 128: 5.5 / 7.9 / 8.6 / 9.3 / 14.1 us so, 6.6 / 9.1 / 9.3 / 7.5 / 10.1 by warps).  The number
// is rounded down to a power of two: with 4, blocks of 6 and 7 would come along, which lose 1.8 us
// where 4 gains 0.7.
constexpr int Q8_FEW = 2;

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

// A lane's two vectors of eight elements of a row of keys or values: weighed and rotated, the
// row's norm left to the factor that makes them codes.  Element e becomes A x_e + B x_e', with e'
// its partner in the rotation, A = w_e cos and B = -+ w_e' sin: both from a table of the block's
// tokens, four floats (A, A, B, B) for two elements, the lanes of a row side by side.  Where pairs
// are halves of whole vectors a lane holds a vector and its partners', else two neighbours.
template <typename E, int L, int MODE>
struct Q8Lane {
  static constexpr int PITCH = 8 * L + (L == 4 ? 4 : 0);  // float4 of a token; rows meet no bank twice
  const AppendArgs& a;
  const float4* s_tab;
  const E* w;       // keys' (or queries') weights, or NULL
  int l, v0, v1;
  bool on, turned;  // it has elements; (halves) they are rotated
  unsigned mates;

  SLS_DEV Q8Lane(const AppendArgs& args, const float4* tab, const void* weight, int lane, int l_)
      : a(args), s_tab(tab), w(reinterpret_cast<const E*>(weight)), l(l_), mates(((1u << L) - 1) << (lane & ~(L - 1))) {
    const int half = MODE == Q8_HALVES ? a.pairs >> 3 : 0;
    turned = l < half;
    v0 = turned ? l : 2 * l;
    v1 = turned ? l + half : 2 * l + 1;
    on = v1 < a.c.head_dim >> 3;
  }

  // Element e of token `slot` in the table: A, and B two floats on.
  SLS_DEV float* entry(float4* tab, int slot, int e) const {
    int lane = e >> 4, at = e & 15;
    if (MODE == Q8_HALVES && e < 2 * a.pairs) {
      const bool low = e < a.pairs;
      lane = (low ? e : e - a.pairs) >> 3;
      at = (low ? 0 : 8) + (e & 7);
    }
    return reinterpret_cast<float*>(tab + slot * PITCH + (at >> 1) * L + lane) + (at & 1);
  }
  // The table of n tokens from slot `lo` on, the first of them packed row `row` and cache index x.
  // FAST: by the hardware's sine and cosine, for what becomes codes.
  template <bool FAST>
  SLS_DEV void enter(float4* tab, int lo, int n, int64_t row, int x) const {
    int width = 8;  // a thread keeps to one pair
    while (width < a.pairs) width *= 2;
    const int pr = threadIdx.x & (width - 1);
    if (pr < a.pairs) {
      const int e = MODE == Q8_SIDES ? 2 * pr : pr, o = MODE == Q8_SIDES ? e + 1 : pr + a.pairs;
      const float we = (w ? (float)w[e] : 1.f) * a.rope_scale,
                  wo = (w ? (float)w[o] : 1.f) * a.rope_scale, f = a.inv_freq[pr];
      float* to_e = entry(tab, lo, e);
      float* to_o = entry(tab, lo, o);
#pragma unroll 1
      for (int k = threadIdx.x / width; k < n; k += blockDim.x / width) {
        const int p = a.positions ? a.positions[row + k] : x + k;
        const float2 cs = FAST ? turn_fast(p, f) : turn(p, f);
        to_e[4 * PITCH * k] = cs.x * we, to_e[4 * PITCH * k + 2] = -cs.y * wo;
        to_o[4 * PITCH * k] = cs.x * wo, to_o[4 * PITCH * k + 2] = cs.y * we;
      }
    }
    // elements that are not rotated
#pragma unroll 1
    for (int e = 2 * a.pairs + (threadIdx.x & 15); e < a.c.head_dim; e += 16) {
      const float we = w ? (float)w[e] : 1.f;
#pragma unroll 1
      for (int k = threadIdx.x >> 4; k < n; k += blockDim.x / 16) {
        float* to = entry(tab, lo + k, e);
        to[0] = we, to[2] = 0.f;
      }
    }
  }

  SLS_DEV void load(const char* p, uint4 (&u)[2]) const {
    u[0] = u[1] = make_uint4(0, 0, 0, 0);
    if (!on) return;
    u[0] = *reinterpret_cast<const uint4*>(p + 16 * v0);
    u[1] = *reinterpret_cast<const uint4*>(p + 16 * v1);
  }

  // u: the row at p, loaded; y: its elements without the norm; most: the largest finite size.
  // KEYS: else as it comes.  known: the norm, where it is (and `most` is not wanted).
  template <bool KEYS>
  SLS_DEV float row(const uint4 (&u)[2], const char* p, int slot, float (&y)[16], float& most,
                    const float* known = nullptr) const {
    float norm = 1.f;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      float z[8];
      widen8<E>(u[v], z);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[8 * v + e] = z[e];
    }
    if constexpr (KEYS && MODE != Q8_PLAIN) {
      if (known) {
        norm = *known;
      } else if (w) {
        f32x2_t s = mul2(pk2(y[0], y[1]), pk2(y[0], y[1]));
#pragma unroll
        for (int e = 2; e < 16; e += 2) s = fma2(pk2(y[e], y[e + 1]), pk2(y[e], y[e + 1]), s);
        float s0, s1;
        upk2(s, s0, s1);
        s0 += s1;
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) s0 += __shfl_xor_sync(mates, s0, o);
        norm = rsqrtf(__fmaf_rn(s0, 1.f / (float)a.c.head_dim, a.eps));
      }
      if (on) {
        const float4* tab = s_tab + slot * PITCH + l;
        const int pairs = a.pairs;
        const E* xs = reinterpret_cast<const E*>(p);
#pragma unroll
        for (int e = 0; e < (MODE == Q8_HALVES ? 8 : 16); e += 2) {
          const float4 f = tab[(e / 2) * L];
          const f32x2_t x = pk2(y[e], y[e + 1]);
          f32x2_t r = mul2(x, pk2(f.x, f.y));
          if constexpr (MODE == Q8_HALVES) {
            const float4 g = tab[(e / 2 + 4) * L];
            const f32x2_t z = pk2(y[e + 8], y[e + 9]);
            f32x2_t q = mul2(z, pk2(g.x, g.y));
            if (turned) {
              r = fma2(z, pk2(f.z, f.w), r);
              q = fma2(x, pk2(g.z, g.w), q);
            }
            upk2(q, y[e + 8], y[e + 9]);
          } else if constexpr (MODE == Q8_SIDES) {
            if (16 * l + e < 2 * pairs) r = fma2(pk2(y[e + 1], y[e]), pk2(f.z, f.w), r);
          } else {
            // halves that split vectors: partners are read from the row again
            float z[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int i = 16 * l + e + k, o = i < pairs ? i + pairs : i - pairs;
              z[k] = i < 2 * pairs ? (float)xs[o] : 0.f;
            }
            r = fma2(pk2(z[0], z[1]), pk2(f.z, f.w), r);
          }
          upk2(r, y[e], y[e + 1]);
        }
      }
    }
    float m = fabsf(y[0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) m = fmaxf(m, fabsf(y[e]));
    m *= norm;
    if (!(m <= 3.402823466e38f)) {  // some element is not finite
      m = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = fabsf(y[e] * norm);
        if (x <= 3.402823466e38f) m = fmaxf(m, x);
      }
    }
    most = fmaxf(most, m);
    return norm;
  }

  // This lane's codes of the row at d.
  SLS_DEV void store(char* d, const uint4& c) const {
    if (MODE == Q8_HALVES) {
      *reinterpret_cast<uint2*>(d + 8 * v0) = make_uint2(c.x, c.y);
      *reinterpret_cast<uint2*>(d + 8 * v1) = make_uint2(c.z, c.w);
    } else {
      *reinterpret_cast<uint4*>(d + 16 * l) = c;
    }
  }
  SLS_DEV uint4 codes(const char* d) const {
    if (MODE == Q8_HALVES) {
      const uint2 x = *reinterpret_cast<const uint2*>(d + 8 * v0);
      const uint2 y = *reinterpret_cast<const uint2*>(d + 8 * v1);
      return make_uint4(x.x, x.y, y.x, y.y);
    }
    return *reinterpret_cast<const uint4*>(d + 16 * l);
  }
};

// A block of a sequence, one of its two matrices.
struct Q8Block {
  int blk, lo, hi;       // its slots, the first new one, the one past the last
  int j_first, j_end;    // heads
  const char* rows;      // the packed row of slot 0, head 0
  int64_t token_b, head_b;
  char* codes;           // of slot 0, head 0
  int64_t slot_b, code_head_b;
  float* scales;         // of head 0
  int64_t scale_head;
  bool ints;             // codes are integers
};

SLS_DEV uint4 q8_codes(bool ints, const float (&y)[16], float by) {
  return ints ? to_codes16<I8>(y, by) : to_codes16<E4M3>(y, by);
}
SLS_DEV float q8_scale(bool ints, float most) {
  return ints ? code_scale<I8>(most) : code_scale<E4M3>(most);
}
// Codes of a row that lacks its norm, by = 1 / scale.  One product has both factors, except where they
// leave float32's range together (norm 1 / sqrt(eps) of a row of zeros, by 2^126 of a block of them).
SLS_DEV uint4 q8_row_codes(bool ints, float (&y)[16], float norm, float by) {
  float f = norm * by;
  if (f > 3.402823466e38f) {
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] *= norm;
    f = by;
  }
  return q8_codes(ints, y, f);
}
// One over a scale: a power of two as a rule.
SLS_DEV float q8_over(float s) {
  const int bits = __float_as_int(s);
  return (bits & 0x807fffff) == 0 && bits > 0 && bits < 0x7e800000 ? __int_as_float(0x7f000000 - bits)
                                                                   : 1.f / s;
}
// Codes of earlier tokens in units of a larger scale.
template <typename Lane>
SLS_DEV void q8_again(const Lane& me, bool ints, char* d, float by) {
  float z[16];
  const uint4 u = me.codes(d);
  if (ints) codes_float<I8>(u, z);
  else codes_float<E4M3>(u, z);
  me.store(d, q8_codes(ints, z, by));
}

// The larger sizes of two pairs of elements; a NaN is as if it were not there.
template <typename E>
SLS_DEV uint32_t q8_larger(uint32_t a, uint32_t b) {
  using H = typename std::conditional<std::is_same<E, __half>::value, __half2, __nv_bfloat162>::type;
  const H m = __hmax2(*reinterpret_cast<const H*>(&a), __habs2(*reinterpret_cast<const H*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// Few new tokens: a head is one group's of L lanes, all heads at once.
template <bool KEYS, typename E, int L, int MODE>
SLS_DEV void q8_few(const Q8Lane<E, L, MODE>& me, const Q8Block& b) {
  constexpr int NG = Q8_T / L;
#pragma unroll 1
  for (int j = b.j_first + (int)threadIdx.x / L; j < b.j_end; j += NG) {
    float y[16], most = 0.f, norm = 1.f;
    uint4 u[2];
    const char* const p = b.rows + j * b.head_b;
#pragma unroll 1
    for (int slot = b.lo; slot < b.hi; ++slot) {
      me.load(p + slot * b.token_b, u);
      norm = me.template row<KEYS>(u, p + slot * b.token_b, slot, y, most);
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(me.mates, most, o));
    float* sp = b.scales + j * b.scale_head;
    const float was = b.lo > 0 ? *sp : 0.f;
    const float now = fmaxf(q8_scale(b.ints, most), fabsf(was)), by = q8_over(now);
    char* d = b.codes + j * b.code_head_b;
#pragma unroll 1
    for (int slot = b.lo; slot < b.hi; ++slot) {
      if (b.hi - b.lo > 1) {
        me.load(p + slot * b.token_b, u);
        norm = me.template row<KEYS>(u, p + slot * b.token_b, slot, y, most);
      }
      if (me.on) me.store(d + slot * b.slot_b, q8_row_codes(b.ints, y, norm, by));
    }
    if (me.on && now != was)
#pragma unroll 1
      for (int slot = 0; slot < b.lo; ++slot) q8_again(me, b.ints, d + slot * b.slot_b, was * by);
    __syncwarp(me.mates);  // every lane has read the old scale
    if (me.l == 0 && now != was) *sp = now;
  }
}

// A head is `share` warps', each with a run of every 32 / L tokens, which go over their rows twice:
// for the maximum, and (from the caches) for the codes.  Alone (share 1) a warp waits for no other.
template <bool KEYS, typename E, int L, int MODE>
SLS_DEV void q8_many(const Q8Lane<E, L, MODE>& me, const Q8Block& b, int j, bool live, int share,
                     float (&s_most)[2][Q8_T / 32], int& parity, float* norms) {
  constexpr int AT = 32 / L;  // rows of a warp at a time
  constexpr int AHEAD = 2;    // loaded before the first is worked on
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int step = AT * share, slot0 = (warp & (share - 1)) * AT + lane / L;
  const char* const p = b.rows + j * b.head_b;
  float most = 0.f;
  if (live) {
    uint32_t top[4] = {0u, 0u, 0u, 0u};  // (as they come) pairs of sizes
#pragma unroll 1
    for (int s = slot0; s - lane / L < b.hi; s += AHEAD * step) {
      uint4 u[AHEAD][2];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int slot = s + k * step;
        u[k][0] = u[k][1] = make_uint4(0, 0, 0, 0);
        if (slot >= b.lo && slot < b.hi) me.load(p + slot * b.token_b, u[k]);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int slot = s + k * step;
        if constexpr (KEYS && MODE != Q8_PLAIN) {
          float y[16];
          if (slot >= b.lo && slot < b.hi) {
            const float norm = me.template row<KEYS>(u[k], p + slot * b.token_b, slot, y, most);
            if (me.l == 0) norms[slot] = norm;
          }
        } else {
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            top[0] = q8_larger<E>(top[0], u[k][v].x), top[1] = q8_larger<E>(top[1], u[k][v].y);
            top[2] = q8_larger<E>(top[2], u[k][v].z), top[3] = q8_larger<E>(top[3], u[k][v].w);
          }
        }
      }
    }
    if constexpr (!(KEYS && MODE != Q8_PLAIN)) {
      const float2 f = Half2<E>::widen(q8_larger<E>(q8_larger<E>(top[0], top[1]), q8_larger<E>(top[2], top[3])));
      most = fmaxf(f.x, f.y);
      if (__any_sync(0xffffffffu, most > 3.402823466e38f)) {  // an infinity among them: look again
        most = 0.f;
#pragma unroll 1
        for (int slot = slot0; slot < b.hi; slot += step) {
          uint4 u[2];
          float y[16];
          if (slot < b.lo) continue;
          me.load(p + slot * b.token_b, u);
          me.template row<KEYS>(u, p + slot * b.token_b, slot, y, most);
        }
      }
    }
  }
  most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
  float* const sp = b.scales + j * b.scale_head;
  const float was = live && b.lo > 0 ? *sp : 0.f;
  if (share > 1) {
    // A barrier of the head's warps alone: another's may be at values, whose code is a copy of its own.
    // The old scale is read in front of it, and written behind it.
    if (lane == 0) s_most[parity][warp] = most;
    named_sync(1 + warp / share, 32 * share);
    const float each = s_most[parity][(warp & ~(share - 1)) + (lane & (share - 1))];
    most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(each)));
    parity ^= 1;
  } else {
    __syncwarp();
  }
  if (!live) return;
  const float now = fmaxf(q8_scale(b.ints, most), fabsf(was)), by = q8_over(now);
  char* const d = b.codes + j * b.code_head_b;
#pragma unroll 1
  for (int s = slot0; s - lane / L < b.hi; s += 2 * step) {
    uint4 u[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int slot = s + k * step;
      if (slot >= b.lo && slot < b.hi) me.load(p + slot * b.token_b, u[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int slot = s + k * step;
      if (slot >= b.hi) continue;
      if (slot >= b.lo) {
        float y[16], again = 0.f;
        const float norm = me.template row<KEYS>(u[k], p + slot * b.token_b, slot, y, again, norms + slot);
        if (me.on) me.store(d + slot * b.slot_b, q8_row_codes(b.ints, y, norm, by));
      } else if (me.on && now != was) {
        q8_again(me, b.ints, d + slot * b.slot_b, was * by);
      }
    }
  }
  if (slot0 == 0 && me.l == 0 && now != was) *sp = now;
  __syncwarp();  // the norms are read
}

// The queries of packed rows [t, t_end), from the sequence of row t on: a group of lanes for each
// head, a token at a time.
template <int MODE, typename E, int L>
SLS_DEV void q8_queries(const Q8Lane<E, L, MODE>& me, float4* tab, int64_t t, int64_t t_end, int seq) {
  const AppendArgs& a = me.a;
  const CacheView& c = a.c;
#pragma unroll 1
  for (int64_t row = t; row < t_end; ++row) {
    // the cache index, which turns where no positions are given: -1 outside every sequence
    while (a.cu && seq < c.B && a.cu[seq + 1] <= row) ++seq;
    if (!a.cu) seq = (int)row;
    int64_t x = -1;
    if (seq < c.B) x = a.cu ? (int64_t)c.kv_lens[seq] - a.cu[seq + 1] + row : (int64_t)c.kv_lens[seq] - 1;
    if (a.cu && seq < c.B && row < a.cu[seq]) x = -1;
    if (MODE != Q8_PLAIN) {
      __syncthreads();
      me.template enter<false>(tab, 0, 1, row, (int)x);
      __syncthreads();
    }
#pragma unroll 1
    for (int h = (int)threadIdx.x / L; h < a.q_heads; h += Q8_T / L) {
      const char* p = a.q.data + row * a.q.token_b + h * a.q.head_b;
      uint4 u[2];
      float y[16], most = 0.f;
      me.load(p, u);
      const float norm = me.template row<true>(u, p, 0, y, most);
      if (MODE == Q8_ODD) __syncwarp(me.mates);  // partners are read before a row is written in place
      if (!me.on) continue;
      char* d = a.out.data + row * a.out.token_b + h * a.out.head_b;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = y[8 * v + e] * norm;
        *reinterpret_cast<uint4*>(d + 16 * (v ? me.v1 : me.v0)) = narrow8<E>(z);
      }
    }
  }
}

// E: input type; L: lanes of a row (16 elements each); FEW: blocks take few new tokens; MODE: of
// keys.  Jobs are the heads of keys, then those of values.  Rows as they come leave registers for
// three CTAs an SM (10717 tokens of 5 heads of 64, the call 21.8 us with two, 20.6 with three); keys
// that are turned spill there (21345 tokens of 8 heads 119.5 us with two, 144 with three).
template <typename E, int L, bool FEW, int MODE>
__global__ void __launch_bounds__(Q8_T, MODE == Q8_PLAIN && !FEW ? 3 : 2)
kv_append_q8_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ ScaleView sv,
                    int tile, int jobs_per_cta, int share, int query_cta, bool ints) {
  extern __shared__ float4 s_tab[];
  __shared__ float s_most[2][Q8_T / 32];
  __shared__ float s_norm[FEW || MODE == Q8_PLAIN ? 1 : Q8_T / 32][128];  // of a warp's rows
  __shared__ int s_ended[Q8_T / 32];
  const CacheView& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int blk = 1 << sv.shift;
  const int j_first = blockIdx.y * jobs_per_cta;
  const int j_end = min(2 * c.kv_heads, j_first + jobs_per_cta);
  const int64_t t_end = min(a.T, ((int64_t)blockIdx.x + 1) * tile);
  int64_t t = (int64_t)blockIdx.x * tile;

  at_wait_ahead();
  at_go();
  const Q8Lane<E, L, MODE> me(a, s_tab, a.k_weight, lane, threadIdx.x % L);
  int seq = (int)t;
  if (a.cu) {
    int ended = 0;
#pragma unroll 1
    for (int b = threadIdx.x; b < c.B; b += Q8_T) ended += a.cu[b + 1] <= t;
    ended = __reduce_add_sync(0xffffffffu, ended);
    if (lane == 0) s_ended[warp] = ended;
    __syncthreads();
    seq = 0;
    for (int w = 0; w < Q8_T / 32; ++w) seq += s_ended[w];
  }
  if constexpr (FEW) {  // the last CTA of a tile has all queries
    if ((int)blockIdx.y == query_cta) {
      q8_queries<MODE>(Q8Lane<E, L, MODE>(a, s_tab, a.q_weight, lane, threadIdx.x % L), s_tab, t, t_end, seq);
      return;
    }
  }
  int parity = 0;
#pragma unroll 1
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
#pragma unroll 1
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
      // the factors of the block's new tokens, for all heads of keys
      if (MODE != Q8_PLAIN && j_first < c.kv_heads) {
        __syncthreads();
        me.template enter<true>(s_tab, lo, hi - lo, row0 + lo, (int)(start + lo));
        __syncthreads();
      }
      const int64_t at_codes = page * c.page_b + slot0 * c.slot_b;
      const Q8Block k{blk, lo, hi, j_first, min(j_end, c.kv_heads),
                      a.k.data + row0 * a.k.token_b, a.k.token_b, a.k.head_b,
                      c.k + at_codes, c.slot_b, c.head_b, sv.k + sc, sv.head, ints};
      const Q8Block v{blk, lo, hi, max(0, j_first - c.kv_heads), j_end - c.kv_heads,
                      a.v.data + row0 * a.v.token_b, a.v.token_b, a.v.head_b,
                      c.v + at_codes, c.slot_b, c.head_b, sv.v + sc, sv.head, ints};
      if constexpr (FEW) {
        q8_few<true>(me, k);
        q8_few<false>(me, v);
      } else {
        const int together = Q8_T / 32 / share;
#pragma unroll 1
        for (int j0 = j_first; j0 < j_end; j0 += together) {
          const int j = j0 + warp / share;
          const bool live = j < j_end;
          float* const norms = s_norm[MODE == Q8_PLAIN ? 0 : warp];
          if (j < c.kv_heads) q8_many<true>(me, k, live ? j : 0, live, share, s_most, parity, norms);
          else q8_many<false>(me, v, live ? j - c.kv_heads : 0, live, share, s_most, parity, norms);
        }
      }
    }
  }
}

// Packed tokens of a CTA: a block's, or as many as a sequence has new ones on average.
int q8_tile(const AppendArgs& a, int blk) {
  int tile = blk;
  while (tile > 1 && a.T < (int64_t)tile * a.c.B) tile /= 2;
  return tile;
}

template <typename E, int L, int MODE>
int launch(const AppendArgs& a, const ScaleView& s, bool ints, cudaStream_t stream) {
  const int blk = 1 << s.shift, jobs = 2 * a.c.kv_heads;
  const int tile = q8_tile(a, blk);
  const bool few = tile <= Q8_FEW;
  const int64_t tiles = (a.T + tile - 1) / tile;
  // a warp for a head, or several where that leaves the GPU with less than eight warps an SM
  int share = 1;
  while (share < 8 && share * 32 / L < blk && tiles * jobs * share < Q8_WARPS) share *= 2;
  // jobs that a CTA has in flight, and has in all: every one, shared out where tiles are few
  const int together = few ? Q8_T / L : Q8_T / 32 / share;
  const int passes = (jobs + together - 1) / together;
  const int ctas = few ? 2 : (int)std::max<int64_t>(1, std::min<int64_t>((Q8_CTAS + tiles - 1) / tiles, passes));
  const int per = (jobs + ctas - 1) / ctas;
  const int query_cta = (jobs + per - 1) / per;
  const dim3 grid((unsigned)tiles, (unsigned)(query_cta + few));
  const size_t smem = MODE != Q8_PLAIN ? (size_t)blk * Q8Lane<E, L, MODE>::PITCH * sizeof(float4) : 0;
  auto go = [&](auto kern) {
    if (smem > 48 * 1024)
      SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        (int)smem));
    return at_launch(kern, grid, Q8_T, smem, 1, stream, a, s, tile, per, share, query_cta, ints);
  };
  return few ? go(kv_append_q8_kernel<E, L, true, MODE>) : go(kv_append_q8_kernel<E, L, false, MODE>);
}

template <typename E, int L>
int launch(const AppendArgs& a, const ScaleView& s, bool ints, cudaStream_t stream) {
  const bool few = q8_tile(a, 1 << s.shift) <= Q8_FEW;
  if (a.pairs == 0 && !a.k_weight && !(few && a.q_weight)) return launch<E, L, Q8_PLAIN>(a, s, ints, stream);
  if (a.interleaved) return launch<E, L, Q8_SIDES>(a, s, ints, stream);
  return (a.pairs & 7) == 0 ? launch<E, L, Q8_HALVES>(a, s, ints, stream)
                            : launch<E, L, Q8_ODD>(a, s, ints, stream);
}

template <typename E>
int launch(const AppendArgs& a, const ScaleView& s, int code, cudaStream_t stream) {
  return a.c.head_dim > 64 ? launch<E, 8>(a, s, code == SLS_I8, stream)
                           : launch<E, 4>(a, s, code == SLS_I8, stream);
}

}  // namespace

int launch_qkv_append_q8(const AppendArgs& a, const ScaleView& s, int code, int dtype,
                        cudaStream_t stream) {
  if (a.T == 0) return SLS_OK;
  const int st = dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, s, code, stream)
                                   : launch<__half>(a, s, code, stream);
  if (st != SLS_OK || q8_tile(a, 1 << s.shift) <= Q8_FEW) return st;
  // The queries by the 16-bit append, without keys and values, in the gaps of the launch above:
  // angles are formed once for all heads there.
  AppendArgs only_q = a;
  only_q.c.kv_heads = 0;
  only_q.beside = true;
  return launch_qkv_append(only_q, dtype, stream);
}

}  // namespace sls
