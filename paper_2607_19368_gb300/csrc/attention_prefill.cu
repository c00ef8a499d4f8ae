// Attention of packed new tokens over the paged cache on the 5th-generation tensor
// cores (sm_103a):  O = softmax(scale Q K^T + mask) V, one pass over the keys with the
// running maximum and sum of a softmax.
//
// A query tile is 128 rows: 128 / G tokens of a sequence with all G query heads of a key
// head, which the tensor map's box lays one after the other, so that keys and values are
// read once for the group whatever G is.  A CTA has two query tiles (an item) and goes over
// the keys in steps of 128:
//   S = Q K^T   both operands in shared memory, float32 scores in tensor memory
//   P = 2^(c (S - m) + a constant)  a thread per row, scores and maximum in registers; 16-bit weights over
//               the scores' columns of tensor memory; m is replaced only when weights would
//               grow past 2^8, and the output scaled to it then (exact: the factor is common
//               to a row's weights, their sum and its output)
//   O += P V    weights from tensor memory, values from shared memory as they lie in
//               the cache, float32 output in tensor memory
// Warps: 0-3 and 4-7 the softmax of the two tiles, 8 finds items and copies queries and
// keys, 11 values (TMA, a ring of stages of 128 keys or values), 9 issues all products, 10
// keeps the ring.  The tiles take turns: while one's weights form, the
// other's products run.
//
// Rounding: scores, maxima, sums and outputs are float32; the weights, which the tensor
// cores take in 16 bits, are rounded once each (the sum is of the unrounded ones), the
// output once at the end: on normally distributed inputs of up to 8192 tokens the error
// against 64 bits is 1.4 times that of the output's rounding alone.  The tensor cores add 16
// keys at a time to the float32 output, so that over m keys a further m / 16 roundings of
// 2^-23 may add up.
//
// Bound by the chain softmax -> products -> softmax of a tile: in a trace of an earlier build
// (446 us in the first of these cases) a step of both tiles took 2730 cycles, the products
// 2112 of them.  8192 tokens of 40 + 8 heads of 128: 470 us, 1.46 PFLOP/s, 75% of the measured
// rate of a large matrix product; 2048 tokens of 28 + 4 heads: 33.6 us, 16 steps of the
// longest item.  Keeping hidden values finite and scores of any size costs 3 to 5% of that.
//
// Published methods used: the running maximum and sum (M. Milakov and N. Gimelshein, "Online
// normalizer calculation for softmax", 2018), tiles of keys against resident queries (T. Dao,
// D. Y. Fu, S. Ermon, A. Rudra and C. Re, NeurIPS 2022), two query tiles whose products and
// softmaxes alternate (J. Shah, G. Bikshandi, Y. Zhang, V. Thakkar, P. Ramani and T. Dao,
// NeurIPS 2024).
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "attention_umma.cuh"

namespace sls {

namespace {

__device__ int g_status;  // SLS_ERR_TIMEOUT once a wait gave up

constexpr int AP_BM = 128;             // rows of a query tile: (token, head of the group)
constexpr int AP_BN = 128;             // keys of a step
constexpr int AP_SOFT_WARPS = 8;       // two warpgroups, one per query tile
constexpr int AP_THREADS = 384;        // and one warpgroup of single warps
constexpr int AP_LOAD_WARP = AP_SOFT_WARPS, AP_MMA_WARP = AP_SOFT_WARPS + 1,
              AP_RING_WARP = AP_SOFT_WARPS + 2, AP_VALUE_WARP = AP_SOFT_WARPS + 3;
constexpr int AP_ITEMS = 2;            // item slots
constexpr float AP_LAZY = 8.f;         // log2 of the growth of the maximum that is let pass
// log2 of a factor of all weights, which the division by their sum takes out again.  bf16 has
// range to spare below: weights stay at most 1 with the growth that is let pass, so sums of
// large values overflow no earlier than those of weights under the true maximum.  float16 uses
// its range up to 2^15, so that many small weights next to a large one (2^-25 and less of it,
// which would round to 0) reach the output as they reach the sum.
template <typename E>
constexpr float AP_SHIFT = std::is_same<E, __nv_bfloat16>::value ? -AP_LAZY : 15.f - AP_LAZY;

template <int HD>
struct ApShape {
  static constexpr int HALVES = HD / 64;
  static constexpr int HALF_BYTES = 128 * 128;          // 128 rows of 64 16-bit elements
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  static constexpr int STAGES = HD == 128 ? 4 : 8;
  static constexpr int OUT_BYTES = 32 * 128;            // 64 elements of a warp's 32 rows
  static constexpr size_t SMEM = (size_t)(2 + STAGES) * TILE_BYTES + AP_SOFT_WARPS * OUT_BYTES + 1024;
};

// An item, or a piece of one: key steps, keys and limits count from key k0.
struct ApItem {
  int seq;            // -1: no more items
  int head;           // key head
  int tok0;           // first packed token of the pair of tiles
  int ntok;           // tokens of the pair
  int tiles[2];       // key steps of each query tile
  int len;            // cached tokens of the sequence
  int lim0;           // keys that the pair's first token sees, before cutting to [0, len]
  int causal;
  int k0;             // a multiple of AP_BN
  int slot;           // where a piece leaves its sums; -1: the item is whole
};

// Few items with many keys: the steps of all items form one list that the CTAs share
// evenly; an item that falls to several CTAs is left in pieces, at most two a CTA (its
// first and its last), and joined by a second launch.
struct ApSplit {
  float2* ml;   // (slot, row of the pair): maximum of the scores, sum of weights
  float4* o;    // (slot, element / 4, row of the pair): unnormalised output
};

// Scores beyond this (in log2 units) are brought to their maximum before they are scaled: the
// rounding of scale times maximum, common to a row's weights, would grow past the range of the
// weights (and, where the maximum changes, past their precision).  Others are scaled and brought
// to it in one fused step, whose share of that rounding is below 2^-14.
constexpr float AP_FAR = 1024.f;

// ---- tcgen05 / TMA wrappers ------------------------------------------------------

SLS_DEV void ap_mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 y;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %6, 0;\n"
      " mov.b64 y, {%2, %5};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(AP_DESC_HI), "r"(lead)
      : "memory");
}
SLS_DEV void ap_st32(uint32_t addr, const float* v) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(v);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(
          addr),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
      "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]),
      "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]),
      "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]),
      "r"(u[29]), "r"(u[30]), "r"(u[31])
      : "memory");
}
SLS_DEV void ap_st16(uint32_t addr, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
      "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]),
      "r"(u[15])
      : "memory");
}
SLS_DEV void ap_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Bounded wait of a whole warp; false when the time is up or another role gave up.
SLS_DEV bool ap_wait(uint64_t* bar, unsigned parity, volatile int* abort_flag) {
  bool ok = mbar_try_wait(bar, parity);
  if (!ok) {
    const long long t0 = clock64();
    for (unsigned it = 0;; ++it) {
      ok = mbar_try_wait(bar, parity);
      if (ok || ((it & 63) == 63 && (*abort_flag || clock64() - t0 > SLS_WAIT_CYCLES))) break;
    }
  }
  return __all_sync(0xffffffffu, ok);
}

// ---- the order of the work ---------------------------------------------------------
// An item is a pair of query tiles (2 * tpt tokens of one sequence, all query heads
// of one key head).  Items go from the longest (most keys) to the shortest, and CTA
// b of g takes numbers b, 2g-1-b, 2g+b, ...: neighbours in the order cost about the
// same, so turning the direction every round evens the sums out.  An item is found
// from its number by a warp without any table: the number of blocks with at least c
// key steps (the level c and above) is a closed form per sequence, summed over the
// sequences by the lanes; a CTA's numbers rise, so its level falls, most often not at
// all or by one.
struct ApOrder {
  const int32_t* cu;
  CacheView c;
  int64_t T;
  int qb;               // tokens of a block
  unsigned qb_mul, qb_shift;  // x / qb = mulhi(x, qb_mul) >> qb_shift for 0 <= x < 2^31
  int causal;
  int level;            // the last item's level
  int at_level, above;  // blocks at the level or above, blocks above it
  int total;            // blocks of all sequences
  int q0, n0, m0;       // this lane's first sequence: first row, new tokens, cached tokens
};

SLS_DEV int ap_div(const ApOrder& o, int x) {
  return (int)(__umulhi((unsigned)x, o.qb_mul) >> o.qb_shift);
}

// first row, new and cached tokens of a sequence, one of this lane's (s % 32 is the lane)
SLS_DEV void ap_lens(const ApOrder& o, int s, int& q0, int& n, int& m) {
  if (s < 32) {
    q0 = o.q0, n = o.n0, m = o.m0;
    return;
  }
  int64_t r0, r1;
  seq_rows(o.cu, s, o.T, r0, r1);
  q0 = (int)r0;
  n = (int)(r1 - r0);
  m = max(o.c.kv_lens[s], 0);
}

// blocks of a sequence whose key steps number at least c
SLS_DEV int ap_count(const ApOrder& o, int n, int m, int c) {
  const int nb = ap_div(o, n + o.qb - 1);
  if (c <= 0) return nb;
  const unsigned x = (unsigned)(c - 1) * AP_BN;  // more than x keys; up to 2^31
  if ((unsigned)m <= x) return 0;
  if (!o.causal) return nb;
  const int e = (int)x - (m - n) + 1;  // the block's last token is number e or later
  return e <= 0 ? nb : nb - min(nb, ap_div(o, e + o.qb - 1) - 1);
}

SLS_DEV int ap_count_all(const ApOrder& o, int c) {
  int sum = 0;
  for (int s = threadIdx.x & 31; s < o.c.B; s += 32) {
    int q0, n, m;
    ap_lens(o, s, q0, n, m);
    sum += ap_count(o, n, m, c);
  }
  return __reduce_add_sync(0xffffffffu, sum);
}

SLS_DEV void ap_order_init(ApOrder& o, const AttnArgs& a, int qb) {
  const int lane = threadIdx.x & 31;
  o.cu = a.cu, o.c = a.c, o.T = a.T, o.qb = qb, o.causal = a.causal;
  // T. Granlund and P. L. Montgomery, "Division by Invariant Integers using
  // Multiplication", 1994: with 2^(l-1) < d <= 2^l, x / d = (x ceil(2^(31+l) / d)) >> (31+l)
  // for x < 2^31 (qb is even, so l >= 1)
  const int l = 32 - __clz(qb - 1);
  o.qb_mul = (unsigned)(((1ull << (31 + l)) + qb - 1) / qb);
  o.qb_shift = l - 1;
  o.q0 = o.n0 = o.m0 = 0;
  if (lane < o.c.B) {
    int64_t r0, r1;
    seq_rows(o.cu, lane, o.T, r0, r1);
    o.q0 = (int)r0;
    o.n0 = (int)(r1 - r0);
    o.m0 = max(o.c.kv_lens[lane], 0);
  }
  int top = o.m0;
  for (int s = 32 + lane; s < o.c.B; s += 32) top = max(top, max(o.c.kv_lens[s], 0));
  // one sequence needs no levels: its blocks go from the last to the first
  o.level = o.c.B == 1 ? 0
                       : (int)(((unsigned)__reduce_max_sync(0xffffffffu, top) + AP_BN - 1) / AP_BN);
  o.above = 0;
  o.at_level = ap_count_all(o, o.level);
  o.total = o.level == 0 ? o.at_level : ap_count_all(o, 0);
}

// a sequence: first row, new tokens, cached tokens, those that the page table can hold
struct ApSeq {
  int q0, n, m, len;
};
SLS_DEV ApSeq ap_seq(const AttnArgs& a, int s) {
  int64_t r0, r1;
  seq_rows(a.cu, s, a.T, r0, r1);
  ApSeq q;
  q.q0 = (int)r0, q.n = (int)(r1 - r0), q.m = max(a.c.kv_lens[s], 0);
  q.len = (int)cache_len(a.c, s);
  return q;
}
// key steps of block b
SLS_DEV int ap_steps(const ApSeq& q, int b, int qb, int causal) {
  const int keys = causal ? q.m - q.n + min((b + 1) * qb, q.n) : q.len;
  return (int)(((unsigned)max(0, min(keys, q.len)) + AP_BN - 1) / AP_BN);
}
// key steps [j0, j1) of block b and a key head, as far as they go
SLS_DEV void ap_item_of(const ApSeq& q, int seq, int b, int head, int j0, int j1, int tpt,
                        int causal, ApItem& it) {
  const int qb = 2 * tpt;
  it.seq = seq, it.head = head, it.causal = causal;
  it.tok0 = q.q0 + b * qb;
  it.ntok = min(qb, q.n - b * qb);
  const int lim0 = causal ? q.m - q.n + b * qb + 1 : q.len;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int nt = min(tpt, it.ntok - t * tpt);  // tokens of the tile
    const int lim = causal ? lim0 + t * tpt + nt - 1 : q.len;
    it.tiles[t] = nt > 0 ? (int)(((unsigned)max(0, min(lim, q.len)) + AP_BN - 1) / AP_BN) : 0;
  }
  // the second tile, unless empty, has the item's last step
  if (it.tiles[1] > 0) it.tiles[1] = max(it.tiles[0], it.tiles[1]);
#pragma unroll
  for (int t = 0; t < 2; ++t) it.tiles[t] = max(0, min(it.tiles[t], j1) - j0);
  it.k0 = j0 * AP_BN;
  it.len = q.len - it.k0;
  it.lim0 = lim0 - it.k0;
  it.slot = -1;
}

// the item number i; false when there is none
SLS_DEV bool ap_find(ApOrder& o, int64_t i, int tpt, ApItem& it) {
  const int heads = o.c.kv_heads;
  if (i >= (int64_t)o.total * heads) return false;
  const int j = (int)i / heads;  // total * heads is below 2^31
  // the highest level with more than j blocks at or above it: down in doubling steps,
  // then halved
  if (j >= o.at_level) {
    int hi = o.level, lo = o.level;  // at hi there are not enough, at lo there will be
    int at_hi = o.at_level, at_lo = o.at_level;
    for (int step = 1; at_lo <= j; step *= 2) {
      hi = lo, at_hi = at_lo;
      lo = max(0, lo - step);
      at_lo = ap_count_all(o, lo);
    }
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1, cnt = ap_count_all(o, mid);
      if (cnt > j) lo = mid, at_lo = cnt;
      else hi = mid, at_hi = cnt;
    }
    o.level = lo, o.at_level = at_lo, o.above = at_hi;
  }
  int left = j - o.above;
  const int lane = threadIdx.x & 31;
  for (int s0 = 0; s0 < o.c.B; s0 += 32) {
    const int s = s0 + lane;
    int q0 = 0, n = 0, m = 0, mine = 0, b0 = 0;
    if (s < o.c.B) {
      ap_lens(o, s, q0, n, m);
      const int ge = ap_count(o, n, m, o.level);
      mine = o.c.B > 1 ? ge - ap_count(o, n, m, o.level + 1) : ge;
      b0 = o.causal ? ap_div(o, n + o.qb - 1) - ge : 0;  // the level's first block
      if (o.c.B == 1) b0 = mine - 1 - 2 * left;          // b0 + left is the block
    }
    int pre = mine;
    if (o.c.B > 1) {
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, pre, d);
        if (lane >= d) pre += x;
      }
    }
    const unsigned hit = __ballot_sync(0xffffffffu, mine > 0 && left < pre);
    if (hit) {
      const int src = __ffs(hit) - 1;
      const int b = __shfl_sync(0xffffffffu, b0 + left - (pre - mine), src);
      q0 = __shfl_sync(0xffffffffu, q0, src);
      n = __shfl_sync(0xffffffffu, n, src);
      m = __shfl_sync(0xffffffffu, m, src);
      ApSeq sq;
      sq.q0 = q0, sq.n = n, sq.m = m;
      sq.len = (int)min((int64_t)m, (int64_t)o.c.max_pages << o.c.page_shift);
      ap_item_of(sq, s0 + src, b, (int)i - j * heads, 0, 0x7fffffff, tpt, o.causal, it);
      return true;
    }
    left -= __shfl_sync(0xffffffffu, pre, 31);
  }
  return false;
}

// ---- the order of the work in split launches ---------------------------------------
// blocks in the order of the tokens, the key heads of a block one after the other

constexpr int AP_LEAST = 4;   // a CTA takes at least so many steps where there are as many
constexpr int AP_GAIN = 10;   // steps that cutting has to save, about what joining costs
// CTAs that share `total` steps, the longest item having `longest`; 0: no item is cut
SLS_DEV int ap_parts(int64_t total, int longest, int most) {
  const int64_t n = (total + AP_LEAST - 1) / AP_LEAST;
  const int parts = (int)(n < most ? n : most);
  return (int64_t)(longest - AP_GAIN) * parts > total ? parts : 0;
}

struct ApWalk {
  ApSeq q;
  int seq, b, head, j;  // the next step
  int64_t left;         // steps still to take
  int taken;            // pieces so far
};

// The warp's first step: number total * cta / parts of the list; false when no item is
// to be cut.
SLS_DEV bool ap_walk_init(ApWalk& w, const AttnArgs& a, int qb) {
  const int lane = threadIdx.x & 31, heads = a.c.kv_heads;
  // steps of one head's items of a sequence
  int longest = 0;
  auto sum_of = [&](int s) {
    int64_t sum = 0;
    if (s < a.c.B) {
      const ApSeq q = ap_seq(a, s);
      for (int b = 0; b * qb < q.n; ++b) {
        const int n = ap_steps(q, b, qb, a.causal);
        sum += n;
        longest = max(longest, n);
      }
    }
    return sum;
  };
  auto scan = [&](int64_t& x) {  // inclusive; returns the warp's sum
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    return __shfl_sync(0xffffffffu, x, 31);
  };
  int64_t total = 0;
  for (int s0 = 0; s0 < a.c.B; s0 += 32) {
    int64_t x = sum_of(s0 + lane);
    total += scan(x);
  }
  total *= heads;
  longest = __reduce_max_sync(0xffffffffu, longest);
  const int parts = ap_parts(total, longest, gridDim.x);
  if (parts == 0) return false;
  w.left = 0, w.taken = 0, w.seq = 0;
  if ((int)blockIdx.x >= parts) return true;
  int64_t at = total * blockIdx.x / parts;
  w.left = total * (blockIdx.x + 1) / parts - at;
  for (int s0 = 0;; s0 += 32) {
    const int64_t mine = sum_of(s0 + lane) * heads;
    int64_t x = mine;
    const int64_t all = scan(x);
    if (at < all) {
      const int src = __ffs(__ballot_sync(0xffffffffu, at < x)) - 1;
      at -= __shfl_sync(0xffffffffu, x - mine, src);
      w.seq = s0 + src;
      break;
    }
    at -= all;
  }
  w.q = ap_seq(a, w.seq);
  for (int b0 = 0;; b0 += 32) {
    const int b = b0 + lane;
    const int64_t mine = b * qb < w.q.n ? (int64_t)ap_steps(w.q, b, qb, a.causal) * heads : 0;
    int64_t x = mine;
    const int64_t all = scan(x);
    if (at < all) {
      const int src = __ffs(__ballot_sync(0xffffffffu, at < x)) - 1;
      at -= __shfl_sync(0xffffffffu, x - mine, src);
      w.b = b0 + src;
      break;
    }
    at -= all;
  }
  const int n = ap_steps(w.q, w.b, qb, a.causal);
  w.head = (int)(at / n);
  w.j = (int)(at - (int64_t)w.head * n);
  return true;
}

// the next item or piece; false when the CTA's share is done
SLS_DEV bool ap_walk(ApWalk& w, const AttnArgs& a, int tpt, ApItem& it) {
  if (w.left == 0) return false;
  const int qb = 2 * tpt;
  int n = ap_steps(w.q, w.b, qb, a.causal);
  if (w.j == n) {  // the next item that has keys
    w.j = 0;
    if (++w.head == a.c.kv_heads) {
      w.head = 0;
      do {
        ++w.b;
        while (w.b * qb >= w.q.n) {
          w.b = 0;
          w.q = ap_seq(a, ++w.seq);
        }
        n = ap_steps(w.q, w.b, qb, a.causal);
      } while (n == 0);
    }
  }
  const int take = (int)min((int64_t)(n - w.j), w.left);
  ap_item_of(w.q, w.seq, w.b, w.head, w.j, w.j + take, tpt, a.causal, it);
  if (take < n) it.slot = 2 * blockIdx.x + (w.taken > 0);
  w.j += take;
  w.left -= take;
  ++w.taken;
  return true;
}

// ---- values that are not finite -------------------------------------------------------
// The tensor cores multiply a hidden key's weight 0 with its value, and 0 times infinity or
// NaN is NaN.  Only the keys from the first token's limit on are hidden from some row of a
// pair of tiles: there (less than 2 * tpt keys, in at most three steps) the ring warp puts 0
// for elements that are not finite before the products read them (ap_clean), and the softmax
// warps add those that a row does see to its finished output (ap_patch).  The rows cost
// nothing of that where all values are finite.

// exponents of all ones in either half of a word: bits 15 and 31
template <typename E>
SLS_DEV uint32_t ap_odd(uint32_t w) {
  constexpr bool BF = std::is_same<E, __nv_bfloat16>::value;
  constexpr uint32_t all = BF ? 0x7f807f80u : 0x7c007c00u, one = BF ? 0x00800080u : 0x04000400u;
  return ((w & all) + one) & 0x80008000u;
}

// Rows [r0, r1) of a tile of values in shared memory (128-byte rows, `halves` blocks of
// them half_bytes apart): 0 for every element that is not finite; true when there was one.
template <typename E, int HALVES>
SLS_DEV bool ap_clean(unsigned char* tile, int half_bytes, int r0, int r1) {
  const int lane = threadIdx.x & 31;
  uint32_t odd = 0;
#pragma unroll 1
  for (int x = r0 * 8 + lane; x < r1 * 8; x += 32)
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const uint4 u = reinterpret_cast<const uint4*>(tile + h * half_bytes)[x];
      odd |= ap_odd<E>(u.x) | ap_odd<E>(u.y) | ap_odd<E>(u.z) | ap_odd<E>(u.w);
    }
  if (!__any_sync(0xffffffffu, odd != 0)) return false;
#pragma unroll 1
  for (int h = 0; h < HALVES; ++h) {
    uint32_t* v = reinterpret_cast<uint32_t*>(tile + h * half_bytes);
#pragma unroll 1
    for (int x = r0 * 32 + lane; x < r1 * 32; x += 32)
      v[x] &= ~((ap_odd<E>(v[x]) >> 15) * 0xffffu);
  }
  return true;
}

// Adds to the finished rows of a warp the elements that ap_clean took out: element e of a
// row that sees key h becomes infinite or NaN as value[h][e] is, and NaN where the key is
// not finite either (its score is then NaN, or an infinity whose weight is NaN or 0).  This
// lane's row sees `keys` keys, the values from h0 on were cleaned, those from h1 on are not
// in this piece; add(row, x) adds x[0..3] to elements 4 lane ... of a row of the warp.
template <typename E, typename Add>
SLS_DEV void ap_patch(const CacheView& c, const ApItem& it, int keys, int h0, int h1, Add add) {
  const int lane = threadIdx.x & 31, e0 = 4 * lane;
  const bool on = e0 < c.head_dim;
  const int mine = min(keys, h1);
  float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    const int64_t at = (int64_t)it.k0 + h;
    const int64_t page = c.table[it.seq * c.table_ld + (at >> c.page_shift)];
    uint2 k = make_uint2(0, 0), v = k;
    if (on && page >= 0 && page < c.num_pages) {
      const int64_t off = page * c.page_b + (at & ((1 << c.page_shift) - 1)) * c.slot_b +
                          it.head * c.head_b + 2 * e0;
      k = *reinterpret_cast<const uint2*>(c.k + off);
      v = *reinterpret_cast<const uint2*>(c.v + off);
    }
    const bool nan = __any_sync(0xffffffffu, (ap_odd<E>(k.x) | ap_odd<E>(k.y)) != 0);
    const float2 a = Half2<E>::widen(v.x), b = Half2<E>::widen(v.y);
    const float w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!(fabsf(w[e]) < INFINITY)) x[e] += nan ? NAN : w[e];
    unsigned rows = __ballot_sync(0xffffffffu, mine == h + 1);  // that see no further key
    if (!__any_sync(0xffffffffu, !(x[0] == 0.f && x[1] == 0.f && x[2] == 0.f && x[3] == 0.f)))
      continue;
    for (; rows; rows &= rows - 1) add(__ffs(rows) - 1, x);
  }
}

// ---- copies of keys or values ----------------------------------------------------------
// One warp's copies into its stages of the ring: K_0 V_0 K_1 V_1 ... of an item, keys at
// even places, values at odd ones.
template <int HD>
struct ApCopy {
  using S = ApShape<HD>;
  const CacheView& c;
  const uint32_t ring;
  uint64_t* full;
  uint64_t* empty;
  volatile int* abort_flag;
  const uint32_t lead;
  const int shift;  // log2 of the slots of one copy: a page, or 128 of them
  const int32_t* table;
  int head, len, k0, nk, page;
  unsigned stage, issued;

  SLS_DEV ApCopy(const CacheView& cache, uint32_t kv, uint64_t* f, uint64_t* e,
                 volatile int* abort)
      : c(cache), ring(kv), full(f), empty(e), abort_flag(abort), lead(at_elect()),
        shift(min(7, cache.page_shift)), table(nullptr), head(0), len(0), k0(0), nk(0), page(-1),
        stage(0), issued(0) {}

  // page numbers of step j: lane l holds that of copy l
  SLS_DEV int page_of(int j) const {
    const int lane = threadIdx.x & 31;
    const int x = j * AP_BN + (lane << shift);
    return (lane < (AP_BN >> shift) && j < nk && x < len) ? table[(k0 + x) >> c.page_shift] : -1;
  }
  SLS_DEV void start(const ApItem& it, int steps) {
    table = c.table + it.seq * c.table_ld;
    head = it.head, len = it.len, k0 = it.k0, nk = steps;
    page = page_of(0);
  }
  // step j of the item, which: 0 keys, 1 values; false when a wait gave up
  SLS_DEV bool step(const CUtensorMap* map, int j, int which) {
    const int next = page_of(j + 1);
    const int copies = (min(AP_BN, len - j * AP_BN) + (1 << shift) - 1) >> shift;  // of each half
    const int slot0 = (k0 + j * AP_BN) & ((1 << c.page_shift) - 1);
    const unsigned at = stage + 2 * j + which, st = at % S::STAGES;
    if (!ap_wait(&empty[st], ((at / S::STAGES) & 1) ^ 1, abort_flag)) return false;
    if (lead) mbar_expect_tx(&full[st], S::HALVES * (copies << shift) * 128);
    __syncwarp();
    uint32_t dst = ring + st * S::TILE_BYTES;
#pragma unroll 1
    for (int i = 0; i < copies; ++i) {
      const int pg = __shfl_sync(0xffffffffu, page, i);
#pragma unroll
      for (int h = 0; h < S::HALVES; ++h)
        at_tma4(lead, dst + h * S::HALF_BYTES, map, 64 * h, slot0, head, pg, &full[st]);
      dst += 128u << shift;
    }
    ++issued;
    page = next;
    return true;
  }
  SLS_DEV void end(int steps) { stage += 2 * steps; }
  // the last copies into each of the warp's stages have landed (the place after the last
  // one's is not known when a wait gave up; every stage's last fill is at most STAGES back)
  SLS_DEV void drain(int which) {
    for (unsigned i = 0; i < S::STAGES / 2; ++i) {
      if (i >= issued) break;
      const unsigned at = 2 * (issued - 1 - i) + which;
      for (unsigned w = 0; w < (1u << 25); ++w)
        if (mbar_try_wait(&full[at % S::STAGES], (at / S::STAGES) & 1)) break;
    }
  }
};

// ---- the kernel --------------------------------------------------------------------
// CUT: items may be cut (a kernel of its own: the search for items is code that runs once an
// item, from beyond the instruction caches)
template <typename E, int HD, bool CUT>
__global__ void __launch_bounds__(AP_THREADS, 1)
attention_prefill_kernel(const __grid_constant__ CUtensorMap tmQ,
                         const __grid_constant__ CUtensorMap tmK,
                         const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ AttnArgs a, const __grid_constant__ ApSplit sp) {
  using S = ApShape<HD>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t q_full[2], q_empty[2], s_full[2], p_half[2], p_full[2], o_full[2], done_bar;
  __shared__ uint64_t kv_full[S::STAGES], kv_empty[S::STAGES];
  __shared__ uint64_t item_full[AP_ITEMS], item_empty[AP_ITEMS];
  __shared__ ApItem s_item[AP_ITEMS];
  // of item k: whether values were cleaned.  A softmax warp may be at the end of an item when
  // the ring warp is two items on (item_empty), so the places are four.
  __shared__ uint64_t clean_full[4];
  __shared__ int s_cleaned[4];
  __shared__ uint32_t tmem_holder;
  __shared__ volatile int s_abort;

  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t q_smem = smem_u32(smem);
  const uint32_t kv_smem = q_smem + 2 * S::TILE_BYTES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = a.q_heads / a.c.kv_heads;
  const int tpt = AP_BM / group;  // tokens of a query tile

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], 1);
      mbar_init(&q_empty[t], 1);
      mbar_init(&s_full[t], 1);
      mbar_init(&p_half[t], AP_SOFT_WARPS / 2 + 1);
      mbar_init(&p_full[t], AP_SOFT_WARPS / 2);
      mbar_init(&o_full[t], 1);
    }
    for (int s = 0; s < S::STAGES; ++s) {
      mbar_init(&kv_full[s], 1);
      mbar_init(&kv_empty[s], 1);
    }
    for (int s = 0; s < AP_ITEMS; ++s) {
      mbar_init(&item_full[s], 1);
      mbar_init(&item_empty[s], AP_SOFT_WARPS + 3);
    }
    for (int s = 0; s < 4; ++s) mbar_init(&clean_full[s], 1);
    mbar_init(&done_bar, 1);
    mbar_fence_init();
    s_abort = 0;
  }
  ApOrder o;
  ApWalk walk;
  bool cut = false;
  ApItem following;
  auto find = [&](unsigned k) {
    following.seq = -1;
    if constexpr (CUT) {
      if (cut) {
        ap_walk(walk, a, tpt, following);
        return;
      }
    }
    ap_find(o, (int64_t)k * gridDim.x + ((k & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x), tpt,
            following);
  };
  if (warp == AP_LOAD_WARP) {
    at_wait_ahead();
    if constexpr (CUT) cut = ap_walk_init(walk, a, 2 * tpt);
    if (!cut) ap_order_init(o, a, 2 * tpt);
    find(0);
  }
  if (warp == AP_MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(&tmem_holder)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  ap_fence_before();
  __syncthreads();
  ap_fence_after();
  at_wait_ahead();
  const uint32_t tmem = tmem_holder;
  // columns of tensor memory: scores (and, over them, weights) of the two tiles, then
  // their outputs

  auto fail = [&]() {
    s_abort = 1;
    atomicExch(&g_status, SLS_ERR_TIMEOUT);
  };

  // registers: 384 x 168 at launch, 2 x 128 x 200 + 128 x 104 from here (208 and 88: 450 us
  // against 441 on 8192 tokens, the copy warp's registers spill)
  if (warp >= AP_SOFT_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");

  if (warp == AP_LOAD_WARP) {
    // ------------------------------ items, queries and keys ------------------------
    ApCopy<HD> cp(a.c, kv_smem, kv_full, kv_empty, &s_abort);
    unsigned q_used[2] = {0, 0};
    bool ok = true;
    for (unsigned k = 0; ok; ++k) {
      const ApItem it = following;
      const unsigned slot = k % AP_ITEMS, use = k / AP_ITEMS;
      if (!ap_wait(&item_empty[slot], (use & 1) ^ 1, &s_abort)) {
        if (lane == 0) fail();
        break;
      }
      if (lane == 0) {
        s_item[slot] = it;
        mbar_arrive(&item_full[slot]);
      }
      if (it.seq < 0) break;
      const int nk = max(it.tiles[0], it.tiles[1]);
      cp.start(it, nk);
      for (int t = 0; t < 2 && ok; ++t) {
        if (it.tiles[t] == 0) continue;
        if (!ap_wait(&q_empty[t], (q_used[t] & 1) ^ 1, &s_abort)) {
          ok = false;
          break;
        }
        ++q_used[t];
        if (cp.lead) mbar_expect_tx(&q_full[t], S::HALVES * group * tpt * 128);
        __syncwarp();
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h)
          at_tma3(cp.lead, q_smem + t * S::TILE_BYTES + h * S::HALF_BYTES, &tmQ, 64 * h,
                  it.head * group, it.tok0 + t * tpt, &q_full[t]);
        if (t == 0 && nk > 0) ok = cp.step(&tmK, 0, 0);
      }
      // (a first tile without keys: its item's first keys are still to come)
      const int begun = it.tiles[0] > 0 ? 1 : 0;
      const int turns = max(nk, 1);
      for (int j = 0; j < turns && ok; ++j) {
        if (j >= begun && j < nk) ok = cp.step(&tmK, j, 0);
        // the next item is looked for while the ring is full
        if (j == min(turns - 1, 1)) find(k + 1);
      }
      if (!ok && lane == 0) fail();
      cp.end(nk);
    }
    // every copy has landed before the CTA may exit
    cp.drain(0);
    for (int t = 0; t < 2; ++t)
      if (q_used[t] > 0)
        for (unsigned w = 0; w < (1u << 25); ++w)
          if (mbar_try_wait(&q_full[t], (q_used[t] - 1) & 1)) break;
  } else if (warp == AP_VALUE_WARP) {
    // ------------------------------ values -----------------------------------------------
    // a warp of their own: short pages make many copies of a step, and a warp issues one in
    // about 100 cycles (a ragged batch in pages of 16: 164 us, 179 with one warp for both; in
    // pages of 128 161 and 158)
    ApCopy<HD> cp(a.c, kv_smem, kv_full, kv_empty, &s_abort);
    bool ok = true;
    for (unsigned k = 0; ok; ++k) {
      const unsigned slot = k % AP_ITEMS;
      if (!ap_wait(&item_full[slot], (k / AP_ITEMS) & 1, &s_abort)) {
        if (lane == 0) fail();
        break;
      }
      const ApItem it = s_item[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_empty[slot]);
      if (it.seq < 0) break;
      const int nk = max(it.tiles[0], it.tiles[1]);
      cp.start(it, nk);
      for (int j = 0; j < nk && ok; ++j) ok = cp.step(&tmV, j, 1);
      if (!ok && lane == 0) fail();
      cp.end(nk);
    }
    cp.drain(1);
  } else if (warp == AP_MMA_WARP) {
    // ------------------------------ products -------------------------------------------
    // One thread for both tiles, so that their turns alternate: while one tile's weights
    // form, the other's products run (a thread for each tile lets both fall into step,
    // and the products wait for the softmax and the softmax for the products).  Little
    // code: its instructions come from beyond the caches that the softmax loops fill.
    const uint32_t lead = at_elect();
    constexpr uint32_t fmt = std::is_same<E, __nv_bfloat16>::value ? 1u : 0u;
    constexpr uint32_t id_common = (1u << 4) | (fmt << 7) | (fmt << 10) |
                                   ((uint32_t)(AP_BM >> 4) << 24);
    constexpr uint32_t id_s = id_common | ((uint32_t)(AP_BN >> 3) << 17);
    constexpr uint32_t id_o = id_common | (1u << 16) | ((uint32_t)(HD >> 3) << 17);
    const uint32_t qd = ap_desc(q_smem, 16);
    const uint32_t kd = ap_desc(kv_smem, 16), vd = ap_desc(kv_smem, S::HALF_BYTES);
    unsigned stage = 0, q_par = 0, p_par = 0;  // ring stages used; a bit for each tile
    bool ok = true;
    auto wait = [&](uint64_t* bar, unsigned parity) {
      ok = ap_wait(bar, parity, &s_abort);
      if (!ok && lead) fail();
      return ok;
    };
    // S = Q K^T of a tile from a ring stage
    auto scores = [&](int t, unsigned st) {
      const uint32_t k = kd + st * (S::TILE_BYTES >> 4), q = qd + t * (S::TILE_BYTES >> 4);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk) {
        const uint32_t off = ((kk >> 2) * S::HALF_BYTES + (kk & 3) * 32) >> 4;
        ap_mma_ss(lead, t * AP_BN, q + off, k + off, id_s, kk > 0);
      }
      ap_commit(lead, &s_full[t]);
    };
    for (unsigned k = 0;; ++k) {
      const unsigned slot = k % AP_ITEMS;
      if (!wait(&item_full[slot], (k / AP_ITEMS) & 1)) break;
      const int seq = __shfl_sync(0xffffffffu, s_item[slot].seq, 0);
      const int n0 = __shfl_sync(0xffffffffu, s_item[slot].tiles[0], 0);
      const int n1 = __shfl_sync(0xffffffffu, s_item[slot].tiles[1], 0);
      const int nk = max(n0, n1);
      __syncwarp();
      if (lead) mbar_arrive(&item_empty[slot]);
      if (seq < 0) break;
      if (nk == 0) continue;
      // the item's ring stages: K_0 V_0 K_1 V_1 ...
      if (!wait(&kv_full[stage % S::STAGES], (stage / S::STAGES) & 1)) break;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if ((t ? n1 : n0) == 0) continue;
        if (!wait(&q_full[t], (q_par >> t) & 1)) break;
        q_par ^= 1u << t;
        ap_fence_after();
        scores(t, stage % S::STAGES);
      }
      if (!ok) break;
#pragma unroll 1
      for (int j = 0; j < nk; ++j) {
        const unsigned sv = (stage + 2 * j + 1) % S::STAGES, sk = (stage + 2 * j + 2) % S::STAGES;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int mine = t ? n1 : n0;
          if (j >= mine) continue;
          // O (+)= P V: the first half of the keys while the weights of the second form
          const uint32_t v = vd + sv * (S::TILE_BYTES >> 4);
          const uint32_t o = 2 * AP_BN + t * HD, w = t * AP_BN;
          if (!wait(&p_half[t], (p_par >> t) & 1)) break;
          ap_fence_after();
#pragma unroll
          for (int kk = 0; kk < AP_BN / 32; ++kk)
            ap_mma_ts(lead, o, w + 8 * kk, v + (2048 >> 4) * kk, id_o, kk > 0 || j > 0);
          if (!wait(&p_full[t], (p_par >> t) & 1)) break;
          p_par ^= 1u << t;
          ap_fence_after();
#pragma unroll
          for (int kk = AP_BN / 32; kk < AP_BN / 16; ++kk)
            ap_mma_ts(lead, o, w + 8 * kk, v + (2048 >> 4) * kk, id_o, 1);
          if (j + 1 < mine) scores(t, sk);
          else ap_commit(lead, &o_full[t]);
        }
        if (!ok) break;
      }
      if (!ok) break;
      stage += 2 * nk;
    }
    // every product issued has completed before tensor memory is freed
    ap_commit(lead, &done_bar);
    for (unsigned w = 0; w < (1u << 25); ++w)
      if (mbar_try_wait(&done_bar, 0)) break;
  } else if (warp == AP_RING_WARP) {
    // ------------------------------ the ring ---------------------------------------------
    // Waits for the keys and values that the products of a step will read, as one more
    // arrival at the weights' barrier, and frees what finished products have read (the
    // second tile's scores of a step come after everything else of it, and speak for
    // both): the product warp waits for nothing but weights, the softmax for nothing but
    // scores.
    unsigned stage = 0, s_par = 0, o_par = 0;  // a bit for each tile
    bool ok = true;
    auto wait = [&](uint64_t* bar, unsigned parity) {
      ok = ap_wait(bar, parity, &s_abort);
      if (!ok && lane == 0) fail();
      return ok;
    };
    for (unsigned k = 0;; ++k) {
      const unsigned slot = k % AP_ITEMS;
      if (!wait(&item_full[slot], (k / AP_ITEMS) & 1)) break;
      const int seq = s_item[slot].seq, len = s_item[slot].len, lim0 = s_item[slot].lim0;
      const int n0 = s_item[slot].tiles[0], n1 = s_item[slot].tiles[1], nk = max(n0, n1);
      // keys from `some` on are hidden from some row of the pair, those from `all` on from all
      const int some = max(0, min(lim0, len));
      const int all = s_item[slot].causal ? min(len, lim0 + s_item[slot].ntok - 1) : len;
      bool cleaned = false;
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_empty[slot]);
      if (seq < 0) break;
      const int last = n1 > 0;  // the tile that speaks for both
      for (int j = 0; j < nk; ++j) {
        const unsigned kst = stage + 2 * j, vst = kst + 1;
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          const int mine = t ? n1 : n0;
          if (j >= mine) continue;
          // the tile's scores of step j are there
          if (!wait(&s_full[t], (s_par >> t) & 1)) break;
          s_par ^= 1u << t;
          if (lane == 0) {
            if (t == last) {
              if (j > 0) mbar_arrive(&kv_empty[(kst - 1) % S::STAGES]);
              mbar_arrive(&kv_empty[kst % S::STAGES]);
            }
            if (j + 1 == mine) mbar_arrive(&q_empty[t]);
          }
          if (!wait(&kv_full[vst % S::STAGES], (vst / S::STAGES) & 1)) break;
          if ((j + 1) * AP_BN > some && (t == 0 || j >= n0)) {
            // hidden values: whatever their slots hold, zero past the pair's last limit,
            // finite between the first token's and that
            unsigned char* va = smem + (2 + vst % S::STAGES) * S::TILE_BYTES;
            const int r0 = min(AP_BN, all - j * AP_BN), first = max(0, some - j * AP_BN);
            if (first < r0) cleaned |= ap_clean<E, S::HALVES>(va, S::HALF_BYTES, first, r0);
#pragma unroll 1
            for (int x = r0 * 8 + lane; x < AP_BN * 8; x += 32)
#pragma unroll
              for (int h = 0; h < S::HALVES; ++h)
                reinterpret_cast<uint4*>(va + h * S::HALF_BYTES)[x] = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
          if (j + 1 < mine && !wait(&kv_full[(vst + 1) % S::STAGES], ((vst + 1) / S::STAGES) & 1))
            break;
          if (lane == 0) mbar_arrive(&p_half[t]);
        }
        if (!ok) break;
      }
      if (!ok) break;
      if (lane == 0) {
        s_cleaned[k & 3] = cleaned;
        mbar_arrive(&clean_full[k & 3]);
      }
      // the last values: after the last tile's outputs
      if (n0 > 0 && last == 1) o_par ^= 1u;  // the first tile's outputs, not waited for
      if (nk > 0) {
        if (!wait(&o_full[last], (o_par >> last) & 1)) break;
        o_par ^= 1u << last;
        if (lane == 0) mbar_arrive(&kv_empty[(stage + 2 * nk - 1) % S::STAGES]);
      }
      stage += 2 * nk;
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ------------------------------ softmax, a row per thread --------------------------
    const int t = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + t * AP_BN + lanes, to = tmem + 2 * AP_BN + t * HD + lanes;
    unsigned char* stage_out = smem + (2 + S::STAGES) * S::TILE_BYTES + warp * S::OUT_BYTES;
    const int tok_in = row / group, head_in = row - tok_in * group;
    const float c = a.scale * 1.4426950408889634f;
    unsigned s_used = 0, o_used = 0;
    bool ok = true;
    for (unsigned k = 0; ok; ++k) {
      const unsigned slot = k % AP_ITEMS;
      if (!ap_wait(&item_full[slot], (k / AP_ITEMS) & 1, &s_abort)) {
        if (lane == 0) fail();
        break;
      }
      const ApItem it = s_item[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_empty[slot]);
      if (it.seq < 0) break;
      const int tok = t * tpt + tok_in;  // within the pair
      const bool live = row < group * tpt && tok < it.ntok;
      const int keys = live ? max(0, min(it.len, it.causal ? it.lim0 + tok : it.len)) : 0;
      const int nk = it.tiles[t];
      // key steps before this one are seen whole by every live row of the warp
      const int least = __reduce_min_sync(0xffffffffu, live ? keys : 0x7fffffff);
      const int whole = least / AP_BN;
      float mx = -INFINITY, l = 0.f;  // the maximum in use, the sum of weights under it
      bool far = false;               // the maximum is beyond AP_FAR
      auto step = [&](int j, auto hidden) {
        if (!ap_wait(&s_full[t], s_used & 1, &s_abort)) return false;
        ++s_used;
        ap_fence_after();
        float s[AP_BN];
#pragma unroll
        for (int q = 0; q < AP_BN / 32; ++q) ap_ld32(ts + 32 * q, s + 32 * q);
        ap_wait_ld<AP_BN>(s);
        if constexpr (decltype(hidden)::value) {
          const int lim = keys - j * AP_BN, sure = least - j * AP_BN;
#pragma unroll
          for (int q = 0; q < AP_BN / 32; ++q) {
            if (32 * (q + 1) <= sure) continue;  // every row sees these
            asm volatile("" ::: "memory");       // a branch, not 32 predicates
#pragma unroll
            for (int e = 32 * q; e < 32 * q + 32; ++e) s[e] = e < lim ? s[e] : -INFINITY;
          }
        }
        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < AP_BN; e += 8)
#pragma unroll
          for (int i = 0; i < 4; ++i) tops[i] = ap_max3(tops[i], s[e + 2 * i], s[e + 2 * i + 1]);
        const float to_mx = fmaxf(mx, fmaxf(ap_max3(tops[0], tops[1], tops[2]), tops[3]));
        // the output is brought to a new maximum only where the old one lets weights
        // grow past 2^AP_LAZY
        const bool grow = mx == -INFINITY ? to_mx > -INFINITY : (to_mx - mx) * c > AP_LAZY;
        if (__any_sync(0xffffffffu, grow || far)) {
          const float f = grow ? at_exp2((mx - to_mx) * c) : 1.f;
          if (grow) mx = to_mx;
          far = live && mx != -INFINITY && fabsf(mx * c) > AP_FAR;
          l *= f;
          if (j > 0) {
#pragma unroll 1
            for (int q = 0; q < HD / 32; ++q) {
              float o[32];
              ap_ld32(to + 32 * q, o);
              ap_wait_ld<32>(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= f;
              ap_st32(to + 32 * q, o);
            }
          }
          if (__any_sync(0xffffffffu, far)) {
            const float m = far ? mx : 0.f;
            const f32x2_t m2 = pk2(-m, -m);
#pragma unroll
            for (int e = 0; e < AP_BN; e += 2)
              upk2(add2(pk2(s[e], s[e + 1]), m2), s[e], s[e + 1]);
          }
        }
        const float base = mx == -INFINITY ? 0.f
                           : far           ? AP_SHIFT<E>
                                           : __fmaf_rn(-mx, c, AP_SHIFT<E>);
        const f32x2_t c2 = pk2(c, c), b2 = pk2(base, base);
        f32x2_t sum[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
        // weights 2^(c (s - mx)) as 16-bit pairs over the scores' columns
#pragma unroll
        for (int q = 0; q < AP_BN / 32; ++q) {
          uint32_t p[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x, y;
            upk2(fma2(pk2(s[32 * q + 2 * e], s[32 * q + 2 * e + 1]), c2, b2), x, y);
            x = at_exp2(x);
            y = at_exp2(y);
            sum[e & 1] = add2(sum[e & 1], pk2(x, y));
            p[e] = Half2<E>::narrow(x, y);
          }
          ap_st16(ts + 16 * q, p);
          if (q == AP_BN / 64 - 1 || q == AP_BN / 32 - 1) {
            ap_wait_st();
            ap_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(q == AP_BN / 64 - 1 ? &p_half[t] : &p_full[t]);
          }
        }
        float sx, sy;
        upk2(add2(sum[0], sum[1]), sx, sy);
        l += sx + sy;
        return true;
      };
      // steps that every live row of the warp sees whole, then the others
      int j = 0;
#pragma unroll 1
      for (; ok && j < min(nk, whole); ++j) ok = step(j, std::false_type());
#pragma unroll 1
      for (; ok && j < nk; ++j) ok = step(j, std::true_type());
      if (!ok && lane == 0) fail();
      if (!ok) break;
      const int64_t gt = it.tok0 + tok;
      const int h = it.head * group + head_in;
      char* out = a.out.data + gt * a.out.token_b + h * a.out.head_b;
      const float inv = keys > 0 ? 1.f / l : 0.f;
      // rows 4 i + lane / 8 of the warp, of which this lane will store 16-byte pieces
      char* dst[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        dst[i] = reinterpret_cast<char*>(__shfl_sync(
            0xffffffffu, reinterpret_cast<unsigned long long>(live ? out : nullptr),
            4 * i + (lane >> 3)));
      if (nk > 0) {
        if (!ap_wait(&o_full[t], o_used & 1, &s_abort)) {
          if (lane == 0) fail();
          break;
        }
        ++o_used;
        ap_fence_after();
      }
      if (!ap_wait(&clean_full[k & 3], (k >> 2) & 1, &s_abort)) {
        if (lane == 0) fail();
        break;
      }
      const bool cleaned = s_cleaned[k & 3];
      // of the cleaned keys, the item's or piece's
      const int h0 = max(0, min(it.lim0, it.len));
      const int h1 = min(min(it.len, it.lim0 + it.ntok - 1), max(it.tiles[0], it.tiles[1]) * AP_BN);
      if (CUT && it.slot >= 0) {
        // a piece: rows next to one another for every four elements
        const int64_t at = (int64_t)it.slot * 2 * AP_BM + t * AP_BM + row;
        sp.ml[at] = make_float2(mx, l);
        float4* po = sp.o + (int64_t)it.slot * (HD / 4) * 2 * AP_BM + t * AP_BM + row;
#pragma unroll 1
        for (int q = 0; q < HD / 32; ++q) {
          float o[32];
          if (nk > 0) {
            ap_ld32(to + 32 * q, o);
            ap_wait_ld<32>(o);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            po[(8 * q + e / 4) * 2 * AP_BM] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
        ap_fence_before();
        if (cleaned) {
          __syncwarp();
          ap_patch<E>(a.c, it, keys, h0, h1, [&](int src, const float(&x)[4]) {
            // element 4 lane of row src of the warp
            float4* p = po + (int64_t)lane * 2 * AP_BM + (src - lane);
            if (4 * lane >= a.c.head_dim) return;
            const float4 v = *p;
            *p = make_float4(v.x + x[0], v.y + x[1], v.z + x[2], v.w + x[3]);
          });
        }
        continue;
      }
      // 64 elements at a time through shared memory, so that a store instruction writes
      // whole 128-byte pieces of four rows (loops, not straight code: it runs once an
      // item, from beyond the instruction caches)
      const f32x2_t inv2 = pk2(inv, inv);
      const int ch = lane & 7;
#pragma unroll 1
      for (int hf = 0; hf < S::HALVES; ++hf) {
#pragma unroll 1
        for (int q = 0; q < 2; ++q) {
          float o[32];
          if (nk > 0) {
            ap_ld32(to + 64 * hf + 32 * q, o);
            ap_wait_ld<32>(o);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            float x[8];
#pragma unroll
            for (int d = 0; d < 8; d += 2) {
              upk2(mul2(pk2(o[e + d], o[e + d + 1]), inv2), x[d], x[d + 1]);
            }
            *reinterpret_cast<uint4*>(stage_out + lane * 128 +
                                      (((4 * q + (e >> 3)) ^ (lane & 7)) << 4)) = narrow8<E>(x);
          }
        }
        __syncwarp();
        const bool on = 64 * hf + 8 * ch < a.c.head_dim;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int rr = 4 * i + (lane >> 3);
          const uint4 v =
              *reinterpret_cast<const uint4*>(stage_out + rr * 128 + ((ch ^ (rr & 7)) << 4));
          if (dst[i] && on) *reinterpret_cast<uint4*>(dst[i] + 128 * hf + 16 * ch) = v;
        }
        __syncwarp();
      }
      ap_fence_before();
      if (cleaned) {
        ap_patch<E>(a.c, it, keys, h0, h1, [&](int src, const float(&x)[4]) {
          char* p = reinterpret_cast<char*>(__shfl_sync(
              0xffffffffu, reinterpret_cast<unsigned long long>(out), src));
          if (4 * lane >= a.c.head_dim) return;
          uint2* u = reinterpret_cast<uint2*>(p + 8 * lane);
          const uint2 w = *u;
          const float2 y = Half2<E>::widen(w.x), z = Half2<E>::widen(w.y);
          *u = make_uint2(Half2<E>::narrow(y.x + x[0], y.y + x[1]),
                          Half2<E>::narrow(z.x + x[2], z.y + x[3]));
        });
      }
    }
  }
  ap_fence_before();
  __syncthreads();
  if (warp == AP_MMA_WARP) {
    ap_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512)
                 : "memory");
  }
}

// Joins the pieces of the items that were cut: a CTA per item and 8 elements, a
// thread per row, the pieces in the order of the keys.  Rows of items that were not cut
// are there already; rows of items without keys become zero here.
constexpr int AP_JOIN = 8;   // elements of a thread
constexpr int AP_FLIGHT = 4;  // pieces in flight
template <typename E, int HD>
__global__ void __launch_bounds__(2 * AP_BM)
attention_prefill_join_kernel(const __grid_constant__ AttnArgs a,
                              const __grid_constant__ ApSplit sp, int ctas) {
  __shared__ int64_t s_sum[2][2 * AP_BM / 32];
  __shared__ int s_longest[2 * AP_BM / 32];
  const int heads = a.c.kv_heads, group = a.q_heads / heads, tpt = AP_BM / group, qb = 2 * tpt;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int b = blockIdx.x / heads;
  const int head = blockIdx.x - b * heads;
  at_go();
  at_wait_ahead();
  // this block's sequence, the steps before it and of all blocks
  int seq = -1, first = b;
  int64_t before = 0, total = 0;
  int longest = 0;
  for (int s = 0, at = 0; s < a.c.B; ++s) {
    const ApSeq q = ap_seq(a, s);
    const int nb = (q.n + qb - 1) / qb;
    if (seq < 0 && b < at + nb) seq = s, first = b - at;
    for (int x = tid; x < nb; x += 2 * AP_BM) {
      const int n = ap_steps(q, x, qb, a.causal);
      total += n;
      longest = max(longest, n);
      if (at + x < b) before += n;
    }
    at += nb;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, d);
    total += __shfl_xor_sync(0xffffffffu, total, d);
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 0) s_sum[0][warp] = before, s_sum[1][warp] = total, s_longest[warp] = longest;
  __syncthreads();
  before = total = 0;
#pragma unroll
  for (int w = 0; w < 2 * AP_BM / 32; ++w) {
    before += s_sum[0][w], total += s_sum[1][w];
    longest = max(longest, s_longest[w]);
  }
  total *= heads;
  const int parts = ap_parts(total, longest, ctas);
  if (seq < 0 || parts == 0) return;
  b = first;
  const ApSeq q = ap_seq(a, seq);
  const int n = ap_steps(q, b, qb, a.causal);
  const int t = tid / AP_BM, row = tid - t * AP_BM;
  const int tok = t * tpt + row / group;  // within the pair
  const bool live = row < group * tpt && b * qb + tok < q.n;
  const int d0 = AP_JOIN * blockIdx.y;
  if (d0 >= a.c.head_dim) return;
  const int64_t gt = q.q0 + b * qb + tok;
  const int h = head * group + row - (row / group) * group;
  char* out = a.out.data + gt * a.out.token_b + h * a.out.head_b;
  if (n == 0) {
    if (live) {
#pragma unroll
      for (int e = 0; e < AP_JOIN; e += 8)
        if (d0 + e < a.c.head_dim)
          *reinterpret_cast<uint4*>(out + 2 * (d0 + e)) = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  const int64_t x0 = before * heads + (int64_t)head * n, x1 = x0 + n;
  // the CTA of step x is the last whose start total * g / parts is at most x
  const int g0 = (int)(((x0 + 1) * parts - 1) / total), g1 = (int)((x1 * parts - 1) / total);
  if (g0 == g1) return;
  // the first piece is its CTA's last unless the CTA starts with it
  const int late = total * g0 / parts < x0;
  const int keys = live ? max(0, min(q.len, a.causal ? q.m - q.n + b * qb + tok + 1 : q.len)) : 0;
  const float c = a.scale * 1.4426950408889634f;
  float top = -INFINITY, sum = 0.f, o[AP_JOIN];
#pragma unroll
  for (int e = 0; e < AP_JOIN; ++e) o[e] = 0.f;
  for (int g = g0; g <= g1; g += AP_FLIGHT) {
    float2 ml[AP_FLIGHT];
    float4 v[AP_FLIGHT][AP_JOIN / 4];
#pragma unroll
    for (int u = 0; u < AP_FLIGHT; ++u) {
      const int64_t slot = 2 * (g + u) + (g + u == g0 ? late : 0);
      ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int x = 0; x < AP_JOIN / 4; ++x) v[u][x] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g + u <= g1 && live) {
        ml[u] = sp.ml[slot * 2 * AP_BM + tid];
#pragma unroll
        for (int x = 0; x < AP_JOIN / 4; ++x)
          v[u][x] = sp.o[(slot * (HD / 4) + d0 / 4 + x) * 2 * AP_BM + tid];
      }
    }
    float to = top;
#pragma unroll
    for (int u = 0; u < AP_FLIGHT; ++u) to = fmaxf(to, ml[u].x);
    const float base = to == -INFINITY ? 0.f : to, f = at_exp2((top - base) * c);
    top = to;
    sum *= f;
#pragma unroll
    for (int e = 0; e < AP_JOIN; ++e) o[e] *= f;
#pragma unroll
    for (int u = 0; u < AP_FLIGHT; ++u) {
      const float w = at_exp2((ml[u].x - base) * c);
      sum += ml[u].y * w;
#pragma unroll
      for (int x = 0; x < AP_JOIN / 4; ++x) {
        o[4 * x] += v[u][x].x * w, o[4 * x + 1] += v[u][x].y * w;
        o[4 * x + 2] += v[u][x].z * w, o[4 * x + 3] += v[u][x].w * w;
      }
    }
  }
  const float inv = keys > 0 ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < AP_JOIN; e += 8) {
    float x[8];
#pragma unroll
    for (int d = 0; d < 8; ++d) x[d] = o[e + d] * inv;
    if (live && d0 + e < a.c.head_dim)
      *reinterpret_cast<uint4*>(out + 2 * (d0 + e)) = narrow8<E>(x);
  }
}

// Items of a launch at most, its CTAs, and whether it may cut items: where there are no more
// items than SMs and the page tables have room for AP_ROOM steps (the lengths decide on the
// device).  Device time, whole / cut: 50 tokens behind 10000 of 28 + 4 heads 108 / 30 us, 2 x 500
// behind 7001 of 24 + 8 heads of 64 73.4 / 59; 1000 tokens alone 20 / 36, which stay whole
// (both sides before launches overlapped: the cut ones' second launch costs less since).
constexpr int AP_ROOM = 16;
struct ApHost {
  int64_t items;
  int grid;
  bool split;
  size_t ml_b, o_b;
};
int ap_host(const CacheView& c, int64_t T, int q_heads, ApHost* h) {
  int dev = 0, sms = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  SLS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int qb = 2 * (AP_BM / (q_heads / c.kv_heads));
  h->items = ((T + qb - 1) / qb + std::min<int64_t>(c.B, T)) * c.kv_heads;
  const int64_t room = (int64_t)c.max_pages << c.page_shift;
  h->split = h->items <= sms && room >= AP_ROOM * AP_BN;
  h->grid = (int)(h->split ? sms : std::min<int64_t>(h->items, sms));
  const size_t rows = (size_t)h->grid * 2 * 2 * AP_BM;
  const int hd = c.head_dim > 64 ? 128 : 64;
  h->ml_b = h->split ? sls_align256(rows * 8) : 0;
  h->o_b = h->split ? sls_align256(rows * hd * 4) : 0;
  return SLS_OK;
}

template <typename E, int HD, bool CUT>
int launch_as(const AttnArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v,
           const ApHost& h, const ApSplit& sp, cudaStream_t stream) {
  static bool set[64] = {};  // per device
  int dev = 0;
  SLS_CUDA_TRY(cudaGetDevice(&dev));
  auto kern = attention_prefill_kernel<E, HD, CUT>;
  if (dev >= 64 || !set[dev]) {
    SLS_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)ApShape<HD>::SMEM));
    if (dev < 64) set[dev] = true;
  }
  const int st = at_launch(kern, dim3((unsigned)h.grid), AP_THREADS, ApShape<HD>::SMEM, 1, stream,
                           q, k, v, a, sp);
  if constexpr (!CUT) {
    return st;
  } else {
    if (st != SLS_OK) return st;
    return at_launch(attention_prefill_join_kernel<E, HD>, dim3((unsigned)h.items, HD / AP_JOIN),
                     2 * AP_BM, 0, 1, stream, a, sp, h.grid);
  }
}

template <typename E, int HD>
int launch(const AttnArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v,
           const ApHost& h, const ApSplit& sp, cudaStream_t stream) {
  return h.split ? launch_as<E, HD, true>(a, q, k, v, h, sp, stream)
                 : launch_as<E, HD, false>(a, q, k, v, h, sp, stream);
}

}  // namespace

size_t attention_prefill_workspace(const CacheView& c, int64_t T, int q_heads) {
  ApHost h;
  if (T == 0 || c.B == 0 || ap_host(c, T, q_heads, &h) != SLS_OK) return 0;
  return h.ml_b + h.o_b;
}

int launch_attention_prefill(const AttnArgs& a, int dtype, void* workspace, cudaStream_t stream) {
  if (a.T == 0 || a.c.B == 0) return SLS_OK;
  const CacheView& c = a.c;
  const int group = a.q_heads / c.kv_heads, tpt = AP_BM / group;
  ApHost h;
  const int st = ap_host(c, a.T, a.q_heads, &h);
  if (st != SLS_OK) return st;
  if (h.items > 0x7fffffff) return SLS_ERR_UNSUPPORTED;
  ApSplit sp;
  sp.ml = (float2*)workspace;
  sp.o = (float4*)((char*)workspace + h.ml_b);
  CUtensorMap q, k, v;
  {
    const cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)a.q_heads, (cuuint64_t)a.T};
    const cuuint64_t strides[2] = {(cuuint64_t)a.q.head_b, (cuuint64_t)a.q.token_b};
    const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tpt};
    if (!at_map(&q, dtype, 3, a.q.data, dims, strides, box)) return SLS_ERR_UNSUPPORTED;
  }
  {
    const int slots = std::min(AP_BN, 1 << c.page_shift);
    if (!at_cache_map(&k, dtype, c, c.k, slots) || !at_cache_map(&v, dtype, c, c.v, slots))
      return SLS_ERR_UNSUPPORTED;
  }
  const bool wide = c.head_dim > 64;
  if (dtype == SLS_BF16)
    return wide ? launch<__nv_bfloat16, 128>(a, q, k, v, h, sp, stream)
                : launch<__nv_bfloat16, 64>(a, q, k, v, h, sp, stream);
  return wide ? launch<__half, 128>(a, q, k, v, h, sp, stream)
              : launch<__half, 64>(a, q, k, v, h, sp, stream);
}

int prefill_status_word(int** word) {
  void* p = nullptr;
  SLS_CUDA_TRY(cudaGetSymbolAddress(&p, g_status));
  *word = (int*)p;
  return SLS_OK;
}

}  // namespace sls
