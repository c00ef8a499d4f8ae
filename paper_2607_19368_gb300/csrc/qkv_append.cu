// New queries and keys normalised for each head and rotated by their positions,
// keys and values appended to the paged cache, in one pass:
//   y = w x / sqrt(mean(x^2) + eps);  pair (a, b) of y turned by t = p f_i.
//
// A copy bound by HBM bandwidth with some ten operations an element on the way.  A CTA
// takes a few tokens and all (or, for few tokens, a share) of their heads: the cosines
// and sines of a token are formed once and serve all of its heads.  A row (token, head)
// is 8 lanes of two 16-byte vectors (4 lanes for heads of up to 64), the vectors chosen
// so that a lane holds both halves of its rotated pairs; weight, cosine and sine are
// multiplied together once and stay in registers while the lane goes from head to head
// of its token, so that an element costs one multiplication, one fused
// multiply-add and the product with the norm.
//
// 21345 tokens of 32 query, 8 key and 8 value heads of 128: 90.2 us, 5.8 TB/s, 85% of a
// plain copy's rate (a lane per vector with the turns read from shared memory for every
// head took 252).  Two rows in flight and six CTAs of 128 threads per SM: four rows 92, eight CTAs 110 (their
// registers spill), loads ahead of the rows at hand 99.  4 single tokens: 3.5 us, the
// chain of dependent loads (lengths, page, row).
#include <algorithm>

#include "attention.cuh"

namespace sls {

namespace {

constexpr int QA_T = 128;
constexpr int QA_ROWS = 2;     // rows in flight per lane
constexpr int QA_MAX_TOKENS = 8;
constexpr int QA_MAX_PAIRS = SLS_MAX_HEAD_DIM / 2;

enum { QA_PAIRED, QA_INTERLEAVED, QA_ODD };  // halves of whole vectors (or no rotation); pairs
                                             // side by side; halves that split vectors

// cos and sin of p * f.  The product is held as a rounded float32 and its exact
// remainder (one fused multiply-add); Cody and Waite's reduction (W. J. Cody and
// W. Waite, "Software Manual for the Elementary Functions", 1980) takes multiples
// of 2 pi off it, 2 pi split into three float32 parts, each the rounding of what
// the previous ones leave: with |p| and |p f| below 2^24 the first step is exact,
// and the angle is right to a few 2^-24, where the rounded product alone is off by
// up to 2^-24 |p f|.  Past 2^24 the same is done in float64 with 2 pi in two parts,
// which holds for |p f| up to 2^50.
SLS_DEV float2 turn(int p, float f) {
  const float q = (float)p;
  const float x = __fmul_rn(q, f);
  float r;
  if (abs((int64_t)p) <= (1 << 24) && fabsf(x) < 0x1p24f) {
    const float rest = __fmaf_rn(q, f, -x);
    const float k = rintf(x * 0.15915494309189535f);
    r = __fmaf_rn(-k, 0x1.921fb6p+2f, x);
    r = __fmaf_rn(-k, -0x1.777a5cp-23f, r);
    r = __fmaf_rn(-k, -0x1.ee59dap-48f, r);
    r += rest;
  } else {
    const double y = __dmul_rn((double)p, (double)f);
    const double rest = __fma_rn((double)p, (double)f, -y);
    const double k = rint(y * 0.15915494309189535);
    double z = __fma_rn(-k, 0x1.921fb54442d18p+2, y);
    z = __fma_rn(-k, 0x1.1a62633145c07p-52, z);
    r = (float)(z + rest);
  }
  float s, c;
  sincosf(r, &s, &c);
  return make_float2(c, s);
}

// The factors of a lane's two vectors for rows of queries or of keys: element e of the
// first becomes f (x c0[e] - x' s0[e]), of the second f (x' c1[e] + x s1[e]), with x and
// x' the elements e of the two vectors and f the row's norm.
struct QaFactors {
  f32x2_t c0[4], s0[4], c1[4], s1[4];
};

// L lanes per row; heads of one token are shared by QA_T / (L tokens) groups of lanes
template <typename E, int L, int MODE>
__global__ void __launch_bounds__(QA_T, 6)
qkv_append_kernel(const __grid_constant__ AppendArgs a, int tokens, int heads_per_cta) {
  __shared__ float2 s_turn[QA_MAX_TOKENS][QA_MAX_PAIRS];  // (cos, sin) * scale
  __shared__ int64_t s_slot[QA_MAX_TOKENS];               // byte offset of the token's slot, or -1
  __shared__ int s_pos[QA_MAX_TOKENS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int nt = (int)min((int64_t)tokens, a.T - t0);
  const CacheView& c = a.c;

  // this lane's token, first head and vectors
  const int groups = QA_T / L;             // a multiple of tokens
  const int per_token = groups / tokens;
  const int grp = threadIdx.x / L, l = threadIdx.x & (L - 1);
  const int tok = grp / per_token, sub = grp - tok * per_token;
  const int64_t t = t0 + tok;
  const int h_first = blockIdx.y * heads_per_cta;
  const int h_end = min(h_first + heads_per_cta, a.q_heads + 2 * c.kv_heads);
  const int nv = c.head_dim >> 3;
  const int half = MODE == QA_PAIRED ? a.pairs >> 3 : 0;
  const bool rotated = l < half;           // QA_PAIRED: the lane holds a rotated pair
  const int v0 = MODE == QA_PAIRED && !rotated ? 2 * l : l;
  const int v1 = MODE == QA_PAIRED ? (rotated ? l + half : 2 * l + 1) : l + L;
  const bool on0 = v0 < nv, on1 = v1 < nv;

  // heads of queries, keys and values of this lane: first, first + per_token, ... < end
  struct Span {
    int first, end;
  };
  auto span = [&](int start, int count) {
    // of the CTA's heads [h_first, h_end) every per_token-th from sub on is this lane's
    const int lo = max(h_first, start), from = lo - h_first;
    const int skip = (sub - from) & (per_token - 1);  // per_token is a power of two
    return Span{lo + skip - start, min(h_end, start + count) - start};
  };
  const Span sq = span(0, a.q_heads), sk = span(a.q_heads, c.kv_heads),
             sv = span(a.q_heads + c.kv_heads, c.kv_heads);
  uint4 x0[QA_ROWS], x1[QA_ROWS];
  auto load = [&](const char* src, int64_t head_b, int h0, int end) {
#pragma unroll
    for (int u = 0; u < QA_ROWS; ++u) {
      const int h = h0 + u * per_token;
      x0[u] = x1[u] = make_uint4(0, 0, 0, 0);
      if (h < end) {
        const char* p = src + h * head_b;
        if (on0) x0[u] = *reinterpret_cast<const uint4*>(p + 16 * v0);
        if (on1) x1[u] = *reinterpret_cast<const uint4*>(p + 16 * v1);
      }
    }
  };
  at_go();
  at_wait_ahead();
  const char* q_src = a.q.data + t * a.q.token_b;
  load(q_src, a.q.head_b, sq.first, tok < nt ? sq.end : 0);  // while the tokens are looked up

  // where each token goes: its sequence is the number of sequences that end at or
  // before it
  for (int i = warp; i < nt; i += QA_T / 32) {
    const int64_t tt = t0 + i;
    int s = (int)tt;
    if (a.cu) {
      int ended = 0;
      for (int b = lane; b < c.B; b += 32) ended += (a.cu[b + 1] <= tt);
      s = __reduce_add_sync(0xffffffffu, ended);
    }
    if (lane == 0) {
      int64_t idx = -1, slot = -1;
      if (s < c.B) {
        const int64_t m = c.kv_lens[s];
        idx = a.cu ? m - (int64_t)a.cu[s + 1] + tt : m - 1;
        if (a.cu && tt < a.cu[s]) idx = -1;  // before the first sequence
        const int64_t col = idx >> c.page_shift;
        if (idx >= 0 && col < c.max_pages) {
          const int64_t page = c.table[s * c.table_ld + col];
          if (page >= 0 && page < c.num_pages)
            slot = page * c.page_b + (idx & ((1 << c.page_shift) - 1)) * c.slot_b;
        }
      }
      s_slot[i] = slot;
      s_pos[i] = a.positions ? a.positions[tt] : (int)idx;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nt * a.pairs; i += QA_T) {
    const int k = i / a.pairs, pr = i - k * a.pairs;
    const float2 cs = turn(s_pos[k], a.inv_freq[pr]);
    s_turn[k][pr] = make_float2(cs.x * a.rope_scale, cs.y * a.rope_scale);
  }
  __syncthreads();
  if (tok >= nt) return;  // whole groups; no barrier follows
  const unsigned mates = (L == 32 ? 0xffffffffu : ((1u << L) - 1)) << (lane & ~(L - 1));
  const int64_t slot = s_slot[tok];
  const float inv_n = 1.f / (float)c.head_dim;

  // weights and turns of this lane's vectors, multiplied together
  auto factors = [&](const E* w, QaFactors& f) {
    float w0[8], w1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w0[e] = w1[e] = 1.f;
    if (w && on0) widen8<E>(*reinterpret_cast<const uint4*>(w + 8 * v0), w0);
    if (w && on1) widen8<E>(*reinterpret_cast<const uint4*>(w + 8 * v1), w1);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if (MODE == QA_PAIRED) {
        float2 ca = make_float2(1.f, 0.f), cb = ca;
        if (rotated) ca = s_turn[tok][8 * l + e], cb = s_turn[tok][8 * l + e + 1];
        f.c0[e >> 1] = pk2(w0[e] * ca.x, w0[e + 1] * cb.x);
        f.s0[e >> 1] = pk2(-w1[e] * ca.y, -w1[e + 1] * cb.y);
        f.c1[e >> 1] = pk2(w1[e] * ca.x, w1[e + 1] * cb.x);
        f.s1[e >> 1] = pk2(w0[e] * ca.y, w0[e + 1] * cb.y);
      } else if (MODE == QA_INTERLEAVED) {
        // the pair (e, e + 1) of a vector: y_e = c w_e x_e - s w_{e+1} x_{e+1}
        const int p0 = 4 * v0 + (e >> 1), p1 = 4 * v1 + (e >> 1);
        const float2 ca = p0 < a.pairs ? s_turn[tok][p0] : make_float2(1.f, 0.f);
        const float2 cb = p1 < a.pairs ? s_turn[tok][p1] : make_float2(1.f, 0.f);
        f.c0[e >> 1] = pk2(w0[e] * ca.x, w0[e + 1] * ca.x);
        f.s0[e >> 1] = pk2(-w0[e + 1] * ca.y, w0[e] * ca.y);
        f.c1[e >> 1] = pk2(w1[e] * cb.x, w1[e + 1] * cb.x);
        f.s1[e >> 1] = pk2(-w1[e + 1] * cb.y, w1[e] * cb.y);
      } else {
        f.c0[e >> 1] = pk2(w0[e], w0[e + 1]);
        f.c1[e >> 1] = pk2(w1[e], w1[e + 1]);
      }
    }
  };
  // one row of queries or keys: norm, rotation, rounding
  auto row = [&](uint4& r0, uint4& r1, const E* w, const QaFactors& f, const char* src) {
    float x[8], y[8];
    widen8<E>(r0, x);
    widen8<E>(r1, y);
    f32x2_t a2[4], b2[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) a2[e] = pk2(x[2 * e], x[2 * e + 1]), b2[e] = pk2(y[2 * e], y[2 * e + 1]);
    float norm = 1.f;
    if (w) {
      f32x2_t q = mul2(a2[0], a2[0]), r = mul2(b2[0], b2[0]);
#pragma unroll
      for (int e = 1; e < 4; ++e) q = fma2(a2[e], a2[e], q), r = fma2(b2[e], b2[e], r);
      float u, v;
      upk2(add2(q, r), u, v);
      float ss = u + v;
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mates, ss, o);
      norm = rsqrtf(__fmaf_rn(ss, inv_n, a.eps));
    }
    const f32x2_t n2 = pk2(norm, norm);
    f32x2_t u2[4], v2[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u2[e] = mul2(a2[e], f.c0[e]);
      v2[e] = mul2(b2[e], f.c1[e]);
      if (MODE == QA_PAIRED) {
        if (rotated) {
          u2[e] = fma2(b2[e], f.s0[e], u2[e]);
          v2[e] = fma2(a2[e], f.s1[e], v2[e]);
        }
      } else if (MODE == QA_INTERLEAVED) {
        if (4 * v0 + e < a.pairs) u2[e] = fma2(pk2(x[2 * e + 1], x[2 * e]), f.s0[e], u2[e]);
        if (4 * v1 + e < a.pairs) v2[e] = fma2(pk2(y[2 * e + 1], y[2 * e]), f.s1[e], v2[e]);
      }
      upk2(mul2(u2[e], n2), x[2 * e], x[2 * e + 1]);
      upk2(mul2(v2[e], n2), y[2 * e], y[2 * e + 1]);
    }
    if (MODE == QA_ODD) {
      // x and y are weighed and normalised; partners are read from the row
      const E* xs = reinterpret_cast<const E*>(src);
#pragma unroll 1
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = 8 * (k ? v1 : v0) + e;
          if (i >= 2 * a.pairs) continue;
          const int j = i < a.pairs ? i + a.pairs : i - a.pairs;
          float p = (float)xs[j];
          if (w) p *= norm * (float)w[j];
          const float2 cs = s_turn[tok][min(i, j)];
          float& z = k ? y[e] : x[e];
          z = i < a.pairs ? z * cs.x - p * cs.y : z * cs.x + p * cs.y;
        }
      }
      __syncwarp(mates);  // partners are read before a row is written in place
    }
    r0 = narrow8<E>(x);
    r1 = narrow8<E>(y);
  };

  const int stride = QA_ROWS * per_token;
  auto store = [&](char* dst, int64_t head_b, int h0, int end) {
#pragma unroll
    for (int u = 0; u < QA_ROWS; ++u) {
      const int h = h0 + u * per_token;
      if (h >= end) break;
      char* d = dst + h * head_b;
      if (on0) *reinterpret_cast<uint4*>(d + 16 * v0) = x0[u];
      if (on1) *reinterpret_cast<uint4*>(d + 16 * v1) = x1[u];
    }
  };
  // rows of queries or of keys; a token without a place keeps its keys to itself
  auto turned = [&](const char* src, int64_t src_b, char* dst, int64_t dst_b, Span sp,
                    const E* w, bool loaded) {
    if (sp.first >= sp.end) return;
    QaFactors f;
    factors(w, f);
    for (int h0 = sp.first; h0 < sp.end; h0 += stride) {
      if (!loaded) load(src, src_b, h0, sp.end);
      loaded = false;
#pragma unroll
      for (int u = 0; u < QA_ROWS; ++u) {
        const int h = h0 + u * per_token;
        if (h >= sp.end) break;
        row(x0[u], x1[u], w, f, src + h * src_b);
      }
      store(dst, dst_b, h0, sp.end);
    }
  };
  turned(q_src, a.q.head_b, a.out.data + t * a.out.token_b, a.out.head_b, sq,
         reinterpret_cast<const E*>(a.q_weight), true);
  if (slot < 0) return;
  turned(a.k.data + t * a.k.token_b, a.k.head_b, c.k + slot, c.head_b, sk,
         reinterpret_cast<const E*>(a.k_weight), false);
  for (int h0 = sv.first; h0 < sv.end; h0 += stride) {
    load(a.v.data + t * a.v.token_b, a.v.head_b, h0, sv.end);
    store(c.v + slot, c.head_b, h0, sv.end);
  }
}

template <typename E>
int launch(const AppendArgs& a, cudaStream_t stream) {
  const int heads = a.q_heads + 2 * a.c.kv_heads;
  const bool narrow = a.c.head_dim <= 64;
  const int groups = QA_T / (narrow ? 4 : 8);
  // tokens of a CTA: as many as give every lane several heads to keep its factors for,
  // fewer where there would be less than 608 CTAs (four for each of 152 SMs, which hold six),
  // down to one whose heads are shared out
  int tokens = QA_MAX_TOKENS;
  while (tokens > 1 && (a.T + tokens - 1) / tokens < 608) tokens /= 2;
  const int64_t tiles = (a.T + tokens - 1) / tokens;
  const int share = (int)std::max<int64_t>(1, std::min<int64_t>(608 / tiles, heads));
  const int least = groups / tokens;  // heads that one pass of a CTA takes
  const int per = std::max((heads + share - 1) / share, std::min(heads, least));
  const dim3 grid((unsigned)tiles, (unsigned)((heads + per - 1) / per));
  const int mode = a.interleaved ? QA_INTERLEAVED : (a.pairs & 7) ? QA_ODD : QA_PAIRED;
#define QA_LAUNCH(L, MODE) \
  return at_launch(qkv_append_kernel<E, L, MODE>, grid, QA_T, 0, 1, stream, a, tokens, per)
  if (narrow) {
    if (mode == QA_PAIRED) QA_LAUNCH(4, QA_PAIRED);
    else if (mode == QA_INTERLEAVED) QA_LAUNCH(4, QA_INTERLEAVED);
    else QA_LAUNCH(4, QA_ODD);
  } else {
    if (mode == QA_PAIRED) QA_LAUNCH(8, QA_PAIRED);
    else if (mode == QA_INTERLEAVED) QA_LAUNCH(8, QA_INTERLEAVED);
    else QA_LAUNCH(8, QA_ODD);
  }
#undef QA_LAUNCH
}

}  // namespace

int launch_qkv_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
  if (a.T == 0) return SLS_OK;
  return dtype == SLS_BF16 ? launch<__nv_bfloat16>(a, stream) : launch<__half>(a, stream);
}

}  // namespace sls
