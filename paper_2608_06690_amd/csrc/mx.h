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

// Largest magnitude of 8 values of a block; not below inf if one is not finite (the order of the bit
// patterns is that of the magnitudes, with inf and then NaN above them).
__device__ __forceinline__ float mx_amax8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return __uint_as_float(m);
}
// The largest of such values over lanes l, l ^ a and l ^ b (that of all four, a and b applied in turn).
template <int A, int B>
__device__ __forceinline__ float mx_max_lanes(float amax) {
  uint32_t m = __float_as_uint(amax);
  m = max(m, (uint32_t)__shfl_xor((int)m, A, 64));
  m = max(m, (uint32_t)__shfl_xor((int)m, B, 64));
  return __uint_as_float(m);
}
// Of lanes l, l ^ 16, l ^ 32 and l ^ 48 (rows of 16 lanes swapped in the vector unit).
__device__ __forceinline__ float mx_max_rows(float amax) {
  uint32_t m = __float_as_uint(amax);
  auto s = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = max(s[0], s[1]);
  s = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return __uint_as_float(max(s[0], s[1]));
}
// silu for a result that is rounded to e4m3 next: the hardware reciprocal (1 ulp) in place of the division
// that the bf16 paths correct to the last bit.
__device__ __forceinline__ float mx_silu(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }
// The block's 8 values as bytes, with amax of the whole block of 32; returns the scale's exponent.
// A block with a value that is not finite holds NaN only.
__device__ __forceinline__ int mx_pack8(const float (&v)[8], float amax, uint32_t& q0, uint32_t& q1) {
  const int e = mx_exponent(amax);
  const float inv = mx_pow2(-e);
  q0 = mx_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  q1 = mx_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
  if (!(amax < INFINITY)) q0 = q1 = 0x7F7F7F7Fu;
  return e;
}

}  // namespace pmpe
