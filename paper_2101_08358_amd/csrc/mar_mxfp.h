// Microscaled 4-bit floats (gfx950): codes and scales, shared by quantisation (mar_mxfp.hip) and scores (mar_mxfp_scores.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

static inline int mx_blocks(int dim) { return dim / 32 + (dim % 32 != 0); }
static inline const char* mx_check_strides(int dim, int64_t codes_stride, int64_t scales_stride) {
  const int64_t blocks = mx_blocks(dim);
  if (codes_stride < 16 * blocks || codes_stride % 16 || codes_stride > (int64_t)1 << 40) return "codes_stride is below 16 bytes a block, no multiple of 16 or above 2^40";
  if (scales_stride < blocks || scales_stride > (int64_t)1 << 40) return "scales_stride is below a byte a block or above 2^40";
  return nullptr;
}

// The code of v times 2^-e, |v| < 8 (a block's own largest magnitude lies in [4, 8)): nearest level, ties to the even code.
__device__ __forceinline__ unsigned mx_code(float v) {
  const float a = fabsf(v);
  const unsigned c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
  return c | (__float_as_uint(v) >> 31) << 3;
}
// The level of a code with its sign.  Codes 2 .. 7 are 1 + 1 bits of a float: exponent 1 .. 3, mantissa.
__device__ __forceinline__ float mx_value(unsigned c) {
  const unsigned m = c & 7u;
  const unsigned bits = m < 2 ? m * 0x3f000000u : 0x3f000000u + (m << 22);
  return __uint_as_float(bits | (c & 8u) << 28);
}
// 2^(byte - 127); 255: NaN.
__device__ __forceinline__ float mx_scale(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
}
