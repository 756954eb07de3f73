// The 8-bit rule shared by the chunk store's records (a3_q8.hip) and the 8-bit pages (a3_paged.hip): per token and KV head the
// scale is the float32 rounding of max|x| / 127 taken in float64 and the code the float64 quotient x / scale rounded half to
// even, so that the integer decision is the same as in a float64 reference; x = code * scale.
#pragma once

#include "a3_internal.h"

namespace {

typedef signed char i8x8 __attribute__((ext_vector_type(8)));
typedef signed char i8x16 __attribute__((ext_vector_type(16), aligned(8)));

__device__ __forceinline__ float q8_scale(double amax) { return (float)(amax / 127.0); }
__device__ __forceinline__ float q8_code(double v, float s) {
  const double r = s > 0.f ? rint(v / (double)s) : 0.0;
  return (float)fmin(fmax(r, -127.0), 127.0);
}

// Codes of 16 doubles.  x * (1 / scale) is within 2^-51 of the quotient, so a division decides only where one comes that close to a
// half (or the scale is 0): one check for all, so that its code is not even fetched otherwise.
__device__ __forceinline__ i8x16 q8_codes(const double (&v)[16], float s) {
  const double inv = 1.0 / (double)s;
  double n[16];
  bool near = !(s > 0.f);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const double q = v[e] * inv;
    n[e] = rint(q);
    near |= fabs(fabs(q - n[e]) - 0.5) < 1e-9;
  }
  i8x16 code;
#pragma unroll
  for (int e = 0; e < 16; ++e) code[e] = (signed char)(int)fmin(fmax(n[e], -127.0), 127.0);
  if (__builtin_expect(near, 0))
#pragma unroll
    for (int e = 0; e < 16; ++e) code[e] = (signed char)(int)q8_code(v[e], s);
  return code;
}

// Codes of 16 floats, the division spared nearly always: n = x * (1 / scale) rounded is at most a step off, and x - n * scale
// formed in one rounding says whether n is the nearest whole number (rounding is monotone and scale / 2 is a float, so a
// rounded remainder below scale / 2 is a true one below it).  Only a remainder that is not below (a tie, a quotient within
// 1e-5 of one, NaN) and scales whose reciprocal a float does not hold take the division.
__device__ __forceinline__ i8x16 q8_codes(const float (&v)[16], float s) {
  const bool normal = s > 1e-30f && s < 1e30f;
  const float inv = normal ? __builtin_amdgcn_rcpf(s) : 0.f, half = normal ? 0.5f * s : -1.f;
  constexpr float kMagic = 12582912.f;                         // 1.5 * 2^23: the sum's low bits are the rounded number
  uint32_t code[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float m = fmaf(v[e], inv, kMagic);
    if (!(fabsf(fmaf(kMagic - m, s, v[e])) < half)) m = kMagic + q8_code((double)v[e], s);
    code[e] = __float_as_uint(m);
  }
  i8x16 q;
#pragma unroll
  for (int e = 0; e < 16; ++e) q[e] = (signed char)code[e];
  return q;
}

}  // namespace
