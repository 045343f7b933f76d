// e4m3 with power-of-two scales: a block of 128 values (of a row) or 128 x 128
// (of a matrix) is held as q = e4m3(v / s), rounded to nearest even, with
// s = 2^x the smallest power of two for which the block's largest finite |v| is
// at most 448 s (448: the largest e4m3 number).  Dividing by s is exact, so a
// block gives the same bits wherever it is quantised, and each value is off by
// at most 2^-4 of itself (2^-10 s below 2^-6 s).  A block of zeros has s = 1.
// x is at least -127.  Infinities and NaN become NaN; the scale is that of the
// block's finite values.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eb {

// Biased exponent (x + 127) of the scale of a block whose largest finite
// magnitude is amax = 1.f 2^y: y - 8 where 1.f <= 1.75, else y - 7.
__device__ __forceinline__ int scale_exponent(float amax) {
  if (amax == 0.f) return 127;
  const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
  return e < 0 ? 0 : e;
}
// 1 / s, a normal number for every exponent above.
__device__ __forceinline__ float inverse_scale(int e8) { return __uint_as_float((uint32_t)(254 - e8) << 23); }
__device__ __forceinline__ float scale_value(int e8) {
  return e8 == 0 ? 0x1p-127f : __uint_as_float((uint32_t)e8 << 23);
}

// Four values of magnitude at most 448, or NaN, to e4m3, the first in the low
// byte.  Infinities are to be NaN before: what the conversion makes of them
// depends on a mode bit.
__device__ __forceinline__ float nan_if_infinite(float v) { return fabsf(v) == INFINITY ? __builtin_nanf("") : v; }
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

}  // namespace eb
