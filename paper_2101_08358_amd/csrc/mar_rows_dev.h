// Rows of fp32, bf16 or fp16 values with any stride and any alignment of their type (gfx950): eight columns at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

template <int TYPE> struct RowType;                        // MAR_DTYPE_*
template <> struct RowType<0> { typedef float T; };
template <> struct RowType<1> { typedef __bf16 T; };
template <> struct RowType<2> { typedef _Float16 T; };

typedef unsigned row_u4 __attribute__((ext_vector_type(4)));
typedef unsigned short row_h8 __attribute__((ext_vector_type(8)));

// The 16-bit values of columns c .. c + 7 of a row of d columns, zeros from column d on, as four words.  Nothing outside the
// row is read: a part that reaches beyond its end takes the row's last eight columns (take8_bits) and shifts them down (place8_bits).
__device__ __forceinline__ row_u4 take8_bits(const void* row, int c, int d) {
  const unsigned short* r = (const unsigned short*)row;
  if (d < 8) {                                             // uniform
    row_h8 h = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e) if (c + e < d) h[e] = r[c + e];
    return __builtin_bit_cast(row_u4, h);
  }
  row_u4 v;
  __builtin_memcpy(&v, r + min(c, d - 8), 16);
  return v;
}
__device__ __forceinline__ row_u4 place8_bits(row_u4 v, int c, int d) {
  if (d < 8) return v;                                     // uniform
  int k = max(c - (d - 8), 0);                             // columns to shift out
  if ((d & 7) == 0) {                                      // uniform: all or nothing
    if (k) v = (row_u4)(0u);
    return v;
  }
  unsigned long long lo = ((unsigned long long)v[1] << 32) | v[0], hi = ((unsigned long long)v[3] << 32) | v[2];
  if (k >= 8) { lo = 0; hi = 0; k = 0; }
  if (k >= 4) { lo = hi; hi = 0; k -= 4; }
  if (k) { lo = (lo >> (16 * k)) | (hi << (64 - 16 * k)); hi >>= 16 * k; }
  return (row_u4){(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}
__device__ __forceinline__ row_u4 load8_bits(const void* row, int c, int d) { return place8_bits(take8_bits(row, c, d), c, d); }
// Columns c .. c + 3 of a row of fp32 values, likewise.
__device__ __forceinline__ row_u4 take4_floats(const float* r, int c, int d) {
  row_u4 v = {0u, 0u, 0u, 0u};
  if (d < 4) {                                             // uniform
#pragma unroll
    for (int e = 0; e < 3; ++e) if (c + e < d) v[e] = __float_as_uint(r[c + e]);
    return v;
  }
  __builtin_memcpy(&v, r + min(c, d - 4), 16);
  return v;
}
__device__ __forceinline__ row_u4 place4_floats(row_u4 w, int c, int d) {
  if (d < 4) return w;                                     // uniform
  const int k = max(c - (d - 4), 0);
  if ((d & 3) == 0) {                                      // uniform
    if (k) w = (row_u4)(0u);
    return w;
  }
  row_u4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = 0u;                                             // w[e + k]
#pragma unroll
    for (int j = e; j < 4; ++j) v[e] = e + k == j ? w[j] : v[e];
  }
  return v;
}
__device__ __forceinline__ void load4_floats(const float* r, int c, int d, float (&v)[4]) {
  const row_u4 w = place4_floats(take4_floats(r, c, d), c, d);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
}
template <int TYPE> __device__ __forceinline__ float bits_to_float(unsigned short b) {
  if (TYPE == 1) return __uint_as_float((unsigned)b << 16);
  return (float)__builtin_bit_cast(_Float16, b);
}
template <int TYPE> __device__ __forceinline__ void load8(const typename RowType<TYPE>::T* row, int c, int d, float (&v)[8]) {
  if constexpr (TYPE == 0) {
    float a[4], b[4];
    load4_floats(row, c, d, a);
    load4_floats(row, c + 4, d, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else {
    const row_u4 w = load8_bits(row, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = bits_to_float<TYPE>((unsigned short)(w[e >> 1] >> (16 * (e & 1))));
  }
}
// Rounds to the nearest (ties to even) and writes columns c .. c + N - 1 that the row has.
template <int TYPE, int N> __device__ __forceinline__ void store_cols(typename RowType<TYPE>::T* row, int c, int d, const float (&v)[N]) {
  typename RowType<TYPE>::T o[N];
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = (typename RowType<TYPE>::T)v[e];
  const int left = d - c;                                  // c + N may pass 2^31
  if (N <= left) { __builtin_memcpy(row + c, o, sizeof(o)); return; }
#pragma unroll
  for (int e = 0; e < N; ++e) if (e < left) row[c + e] = o[e];
}
template <int TYPE> __device__ __forceinline__ void store8(typename RowType<TYPE>::T* row, int c, int d, const float (&v)[8]) {
  store_cols<TYPE, 8>(row, c, d, v);
}
