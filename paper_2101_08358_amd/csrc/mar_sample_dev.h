// Draws from scores (gfx950): ranking keys and integer weights, shared by the kernels of mar_sample.hip.
#pragma once
#include "mar_common.h"
#include "mar_rows_dev.h"
#include "mar_softmax.h"

typedef unsigned long long draw_u64;

// Scores as unsigned integers in their order; 0: the row does not count (NaN, -infinity).  -0 and 0 are one, +infinity is the largest float.
__device__ __forceinline__ unsigned draw_key(float s) {
  if (!(s > -__builtin_inff())) return 0u;
  const unsigned b = __float_as_uint(fminf(s, 3.402823466e38f) + 0.f);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float draw_score(unsigned key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// round(2^(bits + x log2 e)), x <= 0, to 2^-50 of itself: 2^f by its Taylor series, |f| <= 1/2, (f ln 2)^13 / 13! < 2^-52.
__device__ __forceinline__ draw_u64 draw_weight(double x, int bits) {
  const double n = __builtin_rint(x * 1.4426950408889634);
  if (!(n > -70.0)) return 0;                              // bits <= 61
  // log2 e in two parts: x log2 e - n without the rounding of its product
  const double f = __builtin_fma(x, 2.0355273740931033e-17, __builtin_fma(x, 1.4426950408889634, -n));
  double p = 2.5678435993488206e-11;                       // ln2^k / k!, k = 12 .. 0
  p = __builtin_fma(p, f, 4.4455382718708116e-10);
  p = __builtin_fma(p, f, 7.0549116208011233e-09);
  p = __builtin_fma(p, f, 1.0178086009239699e-07);
  p = __builtin_fma(p, f, 1.3215486790144309e-06);
  p = __builtin_fma(p, f, 1.5252733804059841e-05);
  p = __builtin_fma(p, f, 1.5403530393381609e-04);
  p = __builtin_fma(p, f, 1.3333558146428443e-03);
  p = __builtin_fma(p, f, 9.6181291076284772e-03);
  p = __builtin_fma(p, f, 5.5504108664821580e-02);
  p = __builtin_fma(p, f, 2.4022650695910072e-01);
  p = __builtin_fma(p, f, 6.9314718055994531e-01);
  p = __builtin_fma(p, f, 1.0);
  return (draw_u64)__builtin_rint(__builtin_ldexp(p, bits + (int)n));
}

// ceil(part * whole), part in [0, 1), whole < 2^62.
__device__ __forceinline__ draw_u64 draw_share_up(float part, draw_u64 whole) {
  const draw_u64 p = (draw_u64)((double)part * 0x1p64);
  return __umul64hi(p, whole) + (p * whole != 0);
}
__device__ __forceinline__ draw_u64 draw_share_down(float part, draw_u64 whole) {
  return __umul64hi((draw_u64)((double)part * 0x1p64), whole);
}

struct DrawArgs {
  const void* scores; const uint32_t* allowed;
  const float* temperatures; const int32_t* top_ks; const float *top_ps, *min_ps, *uniforms;
  int32_t* ids; float* log_probs; int32_t* num_kept;
  int64_t score_stride, allowed_stride;
  int32_t rows, draws, segments;
  int32_t top_k; float temperature, top_p, min_p;
  draw_u64* mass;      // [queries][segments]
  uint32_t* ties;      // [queries][segments]
};
// A query's parameters with the special values resolved.
struct DrawParams { double inv_temperature; int top_k; float top_p, min_p; };   // top_k 0, top_p 2, min_p 0: off
__device__ __forceinline__ DrawParams draw_params(const DrawArgs& a, int64_t q) {
  const float t = a.temperatures ? a.temperatures[q] : a.temperature, p = a.top_ps ? a.top_ps[q] : a.top_p, m = a.min_ps ? a.min_ps[q] : a.min_p;
  const int k = a.top_ks ? a.top_ks[q] : a.top_k;
  DrawParams r;
  const bool greedy = !(t > 0.f);
  r.inv_temperature = greedy ? 1.0 : 1.0 / (double)t;
  r.top_k = greedy ? 1 : max(k, 0);
  r.top_p = !(p < 1.f) ? 2.f : fmaxf(p, 0.f);
  r.min_p = m > 0.f ? fminf(m, 1.f) : 0.f;
  return r;
}
