// The exponential in 64 bits, for choices that have to be those of 64-bit arithmetic.
#pragma once
#include <hip/hip_runtime.h>

namespace pmpe {

// exp(x) for x <= 0 to about one step of fp64: x = n ln 2 + r, |r| <= ln 2 / 2, the Taylor sum of e^r up to
// r^13 (the next term is below 2^-57), times 2^n. 0 below -745.
__device__ __forceinline__ double exp64(double x) {
  x = fmax(x, -800.0);
  const double n = __builtin_rint(x * 1.4426950408889634);
  double r = __builtin_fma(n, -0.6931471805599453, x);  // ln 2, and what the double nearest to it leaves
  r = __builtin_fma(n, -2.3190468138462996e-17, r);
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
  return __builtin_amdgcn_ldexp(p, (int)n);
}

}  // namespace pmpe
