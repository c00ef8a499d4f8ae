// A paged cache of 8-bit codes: its views, and codes to and from numbers.
#pragma once

#include <cuda_fp8.h>

#include <type_traits>

#include "attention.cuh"

namespace sls {

// A float for each block of a page and key head (strides in floats).
struct ScaleView {
  float* k;
  float* v;
  int64_t page, block, head;
  int shift;  // log2 of a block's slots
};

struct WeightView {
  float* data;
  int64_t page, head;  // strides in floats; a head's slots are contiguous
};

struct I8 {
  static constexpr float MOST = 127.f;
  static constexpr int TOP_EXP = 6, TOP_MANT = 0x7e0000;  // 127 = 2^6 * 1.984375
};
struct E4M3 {
  static constexpr float MOST = 448.f;
  static constexpr int TOP_EXP = 8, TOP_MANT = 0x600000;  // 448 = 2^8 * 1.75
};

// The least power of two s >= 2^-126 with a <= MOST * s (a >= 0, finite), from a's exponent
// and mantissa alone.
template <typename C>
SLS_DEV float code_scale(float a) {
  const int bits = __float_as_int(a);
  const int e = (bits >> 23) - C::TOP_EXP + ((bits & 0x7fffff) > C::TOP_MANT);
  return __int_as_float(max(e, 1) << 23);
}

// Four codes as two pairs of float16, exactly: (0, 1) and (2, 3).  Integers: the byte with its
// sign bit turned is the last one of 1024 + 128 + c, whose last place is 1.
template <typename C>
SLS_DEV void codes_half(uint32_t u, uint32_t& a, uint32_t& b) {
  if constexpr (std::is_same<C, I8>::value) {
    const uint32_t x = u ^ 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    uint32_t p = __byte_perm(x, 0x64646464u, 0x4140), q = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 y = __hsub2(*reinterpret_cast<__half2*>(&p), off);
    const __half2 z = __hsub2(*reinterpret_cast<__half2*>(&q), off);
    a = *reinterpret_cast<const uint32_t*>(&y);
    b = *reinterpret_cast<const uint32_t*>(&z);
  } else {
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n"
        " cvt.rn.f16x2.e4m3x2 %1, hi;\n}\n"
        : "=r"(a), "=r"(b)
        : "r"(u));
  }
}

// Sixteen codes as float32.
template <typename C>
SLS_DEV void codes_float(const uint4& u, float (&x)[16]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t a, b;
    codes_half<C>(w[i], a, b);
    const float2 f = __half22float2(*reinterpret_cast<__half2*>(&a));
    const float2 g = __half22float2(*reinterpret_cast<__half2*>(&b));
    x[4 * i] = f.x, x[4 * i + 1] = f.y, x[4 * i + 2] = g.x, x[4 * i + 3] = g.y;
  }
}

// Four numbers in units of the scale, rounded to codes; larger ones to +-MOST, NaN to NaN or
// (integers) 0.
template <typename C>
SLS_DEV uint32_t to_codes(float a, float b, float c, float d) {
  if constexpr (std::is_same<C, I8>::value) {
    auto one = [](float x) {
      // a NaN becomes 0, an infinity the largest integer
      return (uint32_t)(max(-127, min(127, __float2int_rn(x)))) & 0xffu;
    };
    return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
  } else {
    uint32_t u;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n"
        " cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n mov.b32 %0, {lo, hi};\n}\n"
        : "=r"(u)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return u;
  }
}

template <typename C>
SLS_DEV uint4 to_codes16(const float (&x)[16], float by) {
  uint4 u;
  u.x = to_codes<C>(x[0] * by, x[1] * by, x[2] * by, x[3] * by);
  u.y = to_codes<C>(x[4] * by, x[5] * by, x[6] * by, x[7] * by);
  u.z = to_codes<C>(x[8] * by, x[9] * by, x[10] * by, x[11] * by);
  u.w = to_codes<C>(x[12] * by, x[13] * by, x[14] * by, x[15] * by);
  return u;
}

// ---- launchers (code: SLS_I8 or SLS_E4M3; dtype: SLS_BF16 or SLS_F16) --------------
int launch_qkv_append_q8(const AppendArgs& a, const ScaleView& s, int code, int dtype,
                        cudaStream_t stream);

// Codes of the sequences' pages written out in 16 bits: `out` is the same cache, its own
// pages and page table.
struct ExpandPlan {
  bool compact;    // a page for every entry of the page table, else the cache's own numbers
  int64_t pages;
  size_t table_b, pool_b;  // bytes: page table, and keys or values
};
ExpandPlan cache_expand_plan(const CacheView& c);
int launch_cache_expand(const CacheView& c, const ScaleView& s, int code, int dtype,
                        const ExpandPlan& p, void* workspace, CacheView* out,
                        cudaStream_t stream);

size_t attention_decode_q8_workspace(const CacheView& c, int q_heads);
int launch_attention_decode_q8(const AttnArgs& a, const ScaleView& s, int code, int dtype,
                               void* workspace, cudaStream_t stream);

size_t attention_weights_workspace(const CacheView& c, int64_t T, int q_heads);
// code: SLS_I8, SLS_E4M3, or dtype for a 16-bit cache
int launch_attention_weights(const AttnArgs& a, const ScaleView& s, const WeightView& w, int code,
                             int dtype, void* workspace, cudaStream_t stream);

// The path for few rows a sequence, and whether it is taken.
bool attention_weights_few(const CacheView& c, int64_t T, int q_heads);
size_t attention_weights_few_workspace(const CacheView& c, int64_t T, int q_heads);
int launch_attention_weights_few(const AttnArgs& a, const ScaleView& s, const WeightView& w,
                                 int code, int dtype, void* workspace, cudaStream_t stream);

struct EvictArgs {
  CacheView c;
  ScaleView s;
  WeightView w;
  int keep, first, last;
  int32_t* kept;
  int32_t* lens;  // as c.kv_lens, to be written
};
int launch_cache_evict(const EvictArgs& a, int code, cudaStream_t stream);

}  // namespace sls
