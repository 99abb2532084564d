// Microscaled 4-bit floats (gfx950): codes and scales, shared by quantisation (mar_mxfp.hip) and scores (mar_mxfp_scores.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/marius_hip.h"

static inline int mx_blocks(int dim) { return dim / 32 + (dim % 32 != 0); }
static inline const char* mx_check_strides(int dim, int64_t codes_stride, int64_t scales_stride) {
  const int64_t blocks = mx_blocks(dim);
  if (codes_stride < 16 * blocks || codes_stride % 16 || codes_stride > (int64_t)1 << 40) return "codes_stride is below 16 bytes a block, no multiple of 16 or above 2^40";
  if (scales_stride < blocks || scales_stride > (int64_t)1 << 40) return "scales_stride is below a byte a block or above 2^40";
  return nullptr;
}

// The codes of eight values times 2^-e, |v| < 8 (a block's own largest magnitude lies in [4, 8)): nearest level, ties to the even code.
__device__ __forceinline__ unsigned mx_codes(const float (&v)[8]) {
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], 1.f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], 1.f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], 1.f, 3);
}
// The levels of eight codes with their signs.
__device__ __forceinline__ void mx_values(unsigned c, float (&v)[8]) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = d[0]; v[5] = d[1]; v[6] = e[0]; v[7] = e[1];
}
// 2^(byte - 127); 255: NaN.
__device__ __forceinline__ float mx_scale(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
}

static inline int64_t mx_tiles(int64_t queries) { return (queries + 31) / 32; }

struct MxPlan { bool few; int rt, stripes, parts, tiles_part, grid; };
// Up to 32 queries: workgroups that stay, two a CU, of waves with their own stripes of 32 rt rows.  More: a workgroup a stripe of 256 rt rows
// and part of the queries' tiles: one a CU at a time, estimated by the rounds of workgroups and their tiles, a workgroup's rows and first
// images costing some two tiles.  (1 query of 2,000,000 x 400: 98 us by the first way, 148 by the second; 32 of them: 156 and 190; 32 queries of few or
// narrow rows are as fast by the second: 2,000,000 x 100: 88 and 78.)
//
// rt, 32 rows a lane each, chosen by times of fp32 scores.  Up to 32 queries: 1 where the table is too short for more to fill the device
// (32,000 x 100: 5.0 us with 1, 7.1 with 4; 64,000 x 400: 6.4 with 1, 7.6 with 2), 4 up to 192 columns (1 query, 4,000,000 x 100: 77 with 1, 51 with
// 4; 256,000 x 100: 7.6 and 7.9), 2 beyond, where the rows ahead take most registers and both are alike (32 queries, 40,000 x 400: 18 with 1,
// 15 with 2; 4,000,000 x 400: 173 and 190).  More: 4 reads a quarter of the images
// and of their matrix operands for the same products, 1 has workgroups enough for small calls and more of them loading rows where these are
// most of the bytes, 2 is between them where many queries meet few rows (us with 1, 2 and 4; fp32 queries where nothing is said):
//   999 x 120,007 x 400   192 162 160     256 x 200,000 x 400   102 - 70         256 x 100,000 x 100   24 26 27     64 x 2,000,000 x 64   129 116 121
//   1,000 x 15,000 x 100  20.9 19.4 21.5  1,000 x 20,000 x 400  40.2 36.3 36.8   2,000 x 12,000 x 400  48 44 45     1,000 x 30,000 x 200  42 38 35
//   4-bit queries: 4,096 x 15,000 x 400   49 39 43    2,000 x 30,000 x 200   38 37 31    1,000 x 30,000 x 400   30 30 32    256 x 500,000 x 400   150 133 132
static inline MxPlan mx_plan(const mar_mxfp* p) {
  MxPlan r = {};
  const int64_t tiles = mx_tiles(p->num_queries);
  const int nk = (p->dim + 63) / 64;
  r.few = tiles <= 1;
  if (r.few) {
    r.rt = p->num_rows <= 64 * 1024 ? 1 : (nk <= 3 ? 4 : 2);
    r.stripes = (int)((p->num_rows + 32 * r.rt - 1) / (32 * r.rt));
    r.grid = (r.stripes + 3) / 4 < 512 ? (r.stripes + 3) / 4 : 512;
    return r;
  }
  const bool rows_first = tiles < 8 && nk <= 4, products_first = p->dtype != MAR_DTYPE_MXFP4 && (tiles >= 16 || nk > 4);
  const int64_t units = p->num_rows * tiles / 1024;
  if (rows_first) r.rt = 1;
  else if (products_first) r.rt = tiles >= 16 && units >= 384 && units < 896 ? 2 : (units >= 512 ? 4 : 1);
  else r.rt = units >= (tiles >= 48 ? 1792 : 2048) ? 4 : (tiles >= 48 && units >= 1024 ? 2 : 1);
  r.stripes = (int)((p->num_rows + 256 * r.rt - 1) / (256 * r.rt));
  const int64_t slots = 256;
  int64_t best = INT64_MAX;
  for (int64_t k = 1; k <= tiles && k <= 1024 && k * r.stripes <= 1 << 22; k += 1 + k / 32) {
    const int64_t each = (tiles + k - 1) / k, parts = (tiles + each - 1) / each, cost = (r.stripes * parts + slots - 1) / slots * (each + 2);
    if (cost < best) { best = cost; r.parts = (int)parts; r.tiles_part = (int)each; }
  }
  r.grid = r.stripes * r.parts;
  return r;
}
