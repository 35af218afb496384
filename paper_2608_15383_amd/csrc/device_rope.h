// Rotary positions: sine and cosine of an angle and the rotation of a pair,
// shared by the decoder's kernels and the paged append.
#pragma once

#include "common.h"

namespace emoe {

// cos and sin (fp32) of an angle |x| < 2^31 in fp64: x - n pi/2 with pi/2
// in two terms (the product with the first is exact inside the fma, the second
// leaves n * 2e-33), then the Taylor polynomials to x^17 on [-pi/4, pi/4] (the
// first omitted term is below 1e-16).  The library's pow, sincos and their
// range reduction for any argument kept the few lanes that rotate a token busy
// for most of the 4.2 us of rope_kv_kernel at one token.
__device__ __forceinline__ void rope_cos_sin(double x, float& c, float& s) {
  const double n = rint(x * 0.63661977236758134308);
  double r = fma(-n, 1.5707963267948965580, x);
  r = fma(-n, 6.1232339957367660359e-17, r);
  const double z = r * r;
  double ps = fma(z, 1.0 / 355687428096000.0, -1.0 / 1307674368000.0);
  ps = fma(z, ps, 1.0 / 6227020800.0);
  ps = fma(z, ps, -1.0 / 39916800.0);
  ps = fma(z, ps, 1.0 / 362880.0);
  ps = fma(z, ps, -1.0 / 5040.0);
  ps = fma(z, ps, 1.0 / 120.0);
  ps = fma(z, ps, -1.0 / 6.0);
  const double sn = fma(r * z, ps, r);
  double pc = fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);
  pc = fma(z, pc, 1.0 / 479001600.0);
  pc = fma(z, pc, -1.0 / 3628800.0);
  pc = fma(z, pc, 1.0 / 40320.0);
  pc = fma(z, pc, -1.0 / 720.0);
  pc = fma(z, pc, 1.0 / 24.0);
  pc = fma(z, pc, -0.5);
  const double cn = fma(z, pc, 1.0);
  const int k = (int)n & 3;
  const double a = (k & 1) ? sn : cn, b = (k & 1) ? cn : sn;
  c = (float)((k == 1 || k == 2) ? -a : a);
  s = (float)(k >= 2 ? -b : b);
}

// Rotation of the pair (a, b) by the angle of cosine c and sine s, with the
// roundings spelled out: the prompt's and the step's kernels share them.
__device__ __forceinline__ void rope_pair(float a, float b, float c, float s, uint16_t& ra,
                                          uint16_t& rb) {
  ra = (uint16_t)f32_to_bf16_rne(fmaf(a, c, -(b * s)));
  rb = (uint16_t)f32_to_bf16_rne(fmaf(a, s, b * c));
}

}  // namespace emoe
