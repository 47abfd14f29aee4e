// Values in 8 bits with block scales: e4m3 elements and one power-of-two scale, stored as its
// biased exponent (e8m0), for every 32 consecutive values of a row.
#pragma once
#include "pmpe_internal.h"

namespace pmpe {

// Exponent e of the block scale 2^e: the smallest power of two with amax / 2^e <= 448 (the largest
// e4m3 value), so nothing saturates; within [-126, 120]. 0 for an empty (all zero) or not finite
// block, whose elements are zeros or NaN.
__device__ __forceinline__ int mx_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  if (u == 0 || u >= 0x7F800000u) return 0;
  // 448 = 1.75 * 2^8: a mantissa above 1.75 needs the next power (subnormal amax: below the range)
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, -126);
}
__device__ __forceinline__ float mx_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // |e| <= 126
// Four values of magnitude at most 448 to e4m3 bytes, round to nearest even.
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}

}  // namespace pmpe
