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
// images costing some two tiles.  (32 queries of 4,000,000 x 100: 164 us by the first way, 183 by the second; 1 of them: 57 and 118.)
//
// rt, 32 rows a lane each, chosen by times of fp32 scores.  Up to 32 queries: 1 where the table is too short for more to fill the device
// (32,000 x 100: 5.6 us with 1, 7.0 with 4; 64,000 x 400: 17 with 1, 13 with 2; 256,000 x 100: 9.3 and 8.7), 4 up to 192 columns, 2 beyond:
// the rows ahead are held in registers.  More: 4 reads a quarter of the images and of their matrix operands for the same products, 1 has
// workgroups enough for small calls and more of them loading rows where these are most of the bytes:
//   999 x 120,007 x 400, fp32 queries    209 us with 1, 158 with 4      256 x 200,000 x 400   102 and 70       1,000 x 30,000 x 100   33 and 28
//   256 x 100,000 x 100                   24 and 28                     64 x 60,000 x 100      11 and 14       64 x 2,000,000 x 128  131 and 145
//   1,000 x 30,000 x 400, 4-bit queries   32 and 34                     4,096 x 12,000 x 400   44 and 48       256 x 500,000 x 400   155 and 139
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
  r.rt = !rows_first && p->num_rows * tiles >= (products_first ? 512 * 1024 : 2048 * 1024) ? 4 : 1;
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
