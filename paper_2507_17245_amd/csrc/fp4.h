// The 4-bit form of cache rows: 32 channels share a power of two as scale (a byte e: 2^(e - 127), 255: NaN), each has a sign and one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6. gfx950 converts pairs from and to it, the scale multiplied in (a float of which the exponent counts).
//
// The scale is the smallest that leaves no channel beyond 7 times it: what lies between 6 and 7 goes to 6 with an error no larger than the half gap
// below it. Relative rms error of normal channels with a limit of 6 | 7 | 8 (the exponent of the largest, less 2): 0.1155 | 0.1119 | 0.1150, of channels of
// different size 0.166 | 0.151 | 0.153.
#pragma once
#include "paged.h"

namespace da {

namespace {

constexpr int kScaleLeast = 1, kScaleMost = 252, kScaleNaN = 255;   // (6 * 2^125 is a float, 6 * 2^126 is not)

__device__ inline float scale_value(int e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }   // as the conversions take it

// The scale byte for the largest magnitude of 32 channels (not negative; NaN where one is).
__device__ inline int scale_of(float most) {
  if (!(most < INFINITY)) return kScaleNaN;
  const uint32_t b = __builtin_bit_cast(uint32_t, most);
  return min(max((int)(b >> 23) - 2 + ((b & 0x7fffffu) > 0x600000u), kScaleLeast), kScaleMost);
}
__device__ inline int scale_of(double most) {
  if (!(most < (double)INFINITY)) return kScaleNaN;
  const uint64_t b = __builtin_bit_cast(uint64_t, most);
  return min(max((int)(b >> 52) - 1023 + 127 - 2 + ((b & 0xfffffffffffffull) > 0xc000000000000ull), kScaleLeast), kScaleMost);
}

// Codes of eight channels, the first in the low bits.
__device__ inline uint32_t codes_of(const float* x, int e) {
  const float s = scale_value(e);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}
// A double rounded to a float for another rounding behind it: to the neighbour with an odd last bit where it is none itself.
__device__ inline float to_odd(double x) {
  const float f = (float)x;
  if ((double)f == x || !(__builtin_fabsf(f) < INFINITY)) return f;
  uint32_t b = __builtin_bit_cast(uint32_t, f);
  b -= __builtin_fabs((double)f) > __builtin_fabs(x) ? 1 : 0;
  return __builtin_bit_cast(float, b | 1);
}
__device__ inline uint32_t codes_of(const double* x, int e) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = to_odd(__builtin_ldexp(x[j], 127 - e));
  return codes_of(y, 127);
}

// Eight channels of a row, as values.
template <typename E>
struct Values8;
template <>
struct Values8<bf16> {
  bf16x8 x;
  __device__ Values8(uint32_t c, float s) {
    const bf16x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3)};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = y[j >> 1][j & 1];
  }
};
template <>
struct Values8<float> {
  f32x4 x[2];
  __device__ Values8(uint32_t c, float s) {
    const f32x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3)};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j >> 2][j & 3] = y[j >> 1][j & 1];
  }
};

}  // namespace

}  // namespace da
