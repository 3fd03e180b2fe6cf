// Rows of the pool in 4 bits: the format, and its conversions by the hardware's.
//
// A row of a head is groups of 32 columns.  A value is a sign and a code of the grid
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 (two bits of exponent, one of mantissa), times its
// group's 2^E; column 2 i is the low half of byte i.  E is held as the byte E + 127,
// the matrix cores' own block scale, with one block for the 32 columns of a lane.
// Every value is a bf16 number: E lies in [-125, 125].
#pragma once

#include "device.h"
#include "internal.h"

namespace specmemo {

constexpr uint32_t kKv4Nan = 255;   // scale byte of a group that held an infinity or a NaN

// Scale byte of a group whose largest magnitude is `amax`: the least E with
// amax <= 7 x 2^E (6 is the largest code and takes what lies up to half a step above
// it), so every value is off by at most half a step of its own binade.
__device__ __forceinline__ uint32_t kv4_scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127, E = e - 2 + ((u & 0x7FFFFFu) > 0x600000u);
  if (e == 128) return kKv4Nan;
  return (uint32_t)(min(max(E, -125), 125) + 127);
}
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two values of byte BYTE of a code word.
template <int BYTE>
__device__ __forceinline__ uint32_t kv4_bf16x2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
template <int BYTE>
__device__ __forceinline__ f32x2_t kv4_f32x2(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, BYTE);
}

// Eight columns in bf16 of one code word.
__device__ __forceinline__ uint4 kv4_bf16x8(uint32_t codes, float scale) {
  return uint4{kv4_bf16x2<0>(codes, scale), kv4_bf16x2<1>(codes, scale), kv4_bf16x2<2>(codes, scale), kv4_bf16x2<3>(codes, scale)};
}

}  // namespace specmemo
