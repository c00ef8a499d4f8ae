// The angle of a rotation by position.
#pragma once

#include "attention.cuh"

namespace sls {

// The angle p * f less a multiple of 2 pi.  The product is held as a rounded float32 and its exact
// remainder (one fused multiply-add); Cody and Waite's reduction (W. J. Cody and
// W. Waite, "Software Manual for the Elementary Functions", 1980) takes multiples
// of 2 pi off it, 2 pi split into three float32 parts, each the rounding of what
// the previous ones leave: with |p| and |p f| below 2^24 the first step is exact,
// and the angle is right to a few 2^-24, where the rounded product alone is off by
// up to 2^-24 |p f|.  Past 2^24 the same is done in float64 with 2 pi in two parts,
// which holds for |p f| up to 2^50.
SLS_DEV float turn_angle(int p, float f) {
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
  return r;
}

SLS_DEV float2 turn(int p, float f) {
  float s, c;
  sincosf(turn_angle(p, f), &s, &c);
  return make_float2(c, s);
}

// The same by the hardware's sine and cosine, 2^-21 off at most: for what becomes codes of 8 bits.
SLS_DEV float2 turn_fast(int p, float f) {
  float s, c;
  __sincosf(turn_angle(p, f), &s, &c);
  return make_float2(c, s);
}

}  // namespace sls
