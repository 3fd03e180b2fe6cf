// Pieces of the bf16 attention tile loops: the score maximum, the LDS swizzles
// and the operand types of the transposing loads.
#pragma once

#include "device.h"

namespace specmemo {

// Maximum of a lane's 32 scores as a tree of three-input maxima (16 operations).
__device__ __forceinline__ float tile_max32(const f32x16 (&x)[2]) {
  float t[12];
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const int e = 3 * i;
    t[i] = fmaxf(fmaxf(x[e >> 4][e & 15], x[(e + 1) >> 4][(e + 1) & 15]), x[(e + 2) >> 4][(e + 2) & 15]);
  }
  t[10] = x[1][14];
  t[11] = x[1][15];
  const float u0 = fmaxf(fmaxf(t[0], t[1]), t[2]), u1 = fmaxf(fmaxf(t[3], t[4]), t[5]);
  const float u2 = fmaxf(fmaxf(t[6], t[7]), t[8]), u3 = fmaxf(fmaxf(t[9], t[10]), t[11]);
  return fmaxf(fmaxf(u0, u1), fmaxf(u2, u3));
}

typedef short s16x4_t __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// LDS swizzles (16-byte chunk index c of tile row r).  K rows are read 16 rows
// at a time at one chunk (MFMA A operand): chunk c of row r sits at c ^ (r % 16).
// V rows are read by the transposing load 4 rows x 4 chunks at a time:
// chunk c of row r sits at c ^ 4 (r % 4).
__device__ __forceinline__ int kswz(int r, int c) { return c ^ (r & 15); }
__device__ __forceinline__ int vswz(int r, int c) { return c ^ ((r & 3) << 2); }

}  // namespace specmemo
