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
  // (beyond 1.75 times a power the next one)
  return min(max((int)((__builtin_bit_cast(uint32_t, most) + 0x1fffffu) >> 23) - 2, kScaleLeast), kScaleMost);
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

// Eight channels of a row, as operands of a product.
__device__ inline bf16x8 values_of(uint32_t c, float s) {
  const bf16x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3)};
  bf16x8 x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = y[j >> 1][j & 1];
  return x;
}

// 16 bytes of values.
template <typename E>
struct Values16;
template <>
struct Values16<bf16> {
  static constexpr int CHANNELS = 8;
  typedef uint32_t Codes;
  bf16x8 x;
  __device__ Values16(uint32_t c, float s) : x(values_of(c, s)) {}
  template <bool ONCE>
  __device__ void store(bf16* p) const {
    if constexpr (ONCE) __builtin_nontemporal_store(x, (bf16x8*)p);
    else *(bf16x8*)p = x;
  }
};
template <>
struct Values16<float> {
  static constexpr int CHANNELS = 4;
  typedef uint16_t Codes;
  f32x4 x;
  __device__ Values16(uint32_t c, float s) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
    x = f32x4{lo[0], lo[1], hi[0], hi[1]};
  }
  template <bool ONCE>
  __device__ void store(float* p) const {
    if constexpr (ONCE) __builtin_nontemporal_store(x, (f32x4*)p);
    else *(f32x4*)p = x;
  }
};

}  // namespace

}  // namespace da
