// Scores in 64 bits, as the routing by scores and its backward take them.
#pragma once
#include "common.h"

namespace moe {

// exp(-x), x >= 0 (a NaN gives 0).  x = n ln 2 + r, |r| <= ln 2 / 2, with ln 2 in two parts; exp(-r) by its Taylor series to the 13th
// power, whose next term is below 2^-57.  A third of the library function's instructions, which covers what cannot come here.
__device__ __forceinline__ double exp_minus(double x) {
  x = __builtin_fmin(x, 800.0);                                  // below the least number
  const double n = __builtin_rint(x * 1.4426950408889634074);
  double r = __builtin_fma(-n, 0.693147180559945286227, x);      // ln 2 rounded to 53 bits, and the rest of it
  r = -__builtin_fma(-n, 2.319046813846299558e-17, r);
  double p = 1.0 / 6227020800.0;
  p = __builtin_fma(p, r, 1.0 / 479001600.0);
  p = __builtin_fma(p, r, 1.0 / 39916800.0);
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_amdgcn_ldexp(p, -(int)n);
}
// 1 / d for d in [1, 2^1000): the hardware's estimate and two Newton steps.
__device__ __forceinline__ double reciprocal64(double d) {
  double y = __builtin_amdgcn_rcp(d);
  y = __builtin_fma(y, __builtin_fma(-d, y, 1.0), y);
  return __builtin_fma(y, __builtin_fma(-d, y, 1.0), y);
}
__device__ __forceinline__ double sigmoid64(float l) {
  const double t = exp_minus(__builtin_fabs((double)l)), y = reciprocal64(1.0 + t);
  return l < 0.f ? t * y : y;
}
// exp(l - m), l <= m; 1 for l = m, infinities too, but 0 for l = -inf
__device__ __forceinline__ double exp_below(float l, float m) {
  return l == -__builtin_huge_valf() ? 0.0 : l == m ? 1.0 : exp_minus((double)m - (double)l);
}

}  // namespace moe
