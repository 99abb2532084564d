// Rows of a table to microscaled 4-bit floats and back (gfx950).
//
// 32 columns of a row (a block) share a scale 2^e, e = floor(log2 of the largest magnitude) - 2, held as the byte e + 127; a column
// is a sign and the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code, at most 6: code 0 .. 7, sign in bit 3.
// v 2^-e is exact in fp32 (a subnormal that it leaves is below every threshold), so that the one rounding is the code's.
//
// Both kernels are bound by memory: a thread takes eight columns (32 bytes of fp32 in, 4 bytes of codes out), four neighbouring threads a
// block, whose maximum they exchange among their lanes.  No row has a workgroup of its own: rows are of any number of blocks, and a
// division a workgroup finds where its 64 blocks lie.
#include "mar_common.h"
#include "mar_mxfp.h"
#include "mar_rows_dev.h"
#include "mar_softmax.h"

struct QuantiseArgs {
  const void* x; uint8_t *codes, *scales;
  int64_t x_stride, codes_stride, scales_stride, blocks, first;   // blocks of all rows; first workgroup
  int32_t dim, row_blocks;
};
// Block and row of a thread: four threads a block, 64 blocks a workgroup, the first found by one division for all of it.
struct BlockOf { int64_t row; int b, part; bool in; };
__device__ __forceinline__ BlockOf block_of(int64_t first, int64_t blocks, int row_blocks) {
  const int64_t base = (first + blockIdx.x) * 64, row0 = base / row_blocks;
  const int in = (int)(threadIdx.x >> 2);
  const unsigned local = (unsigned)(base - row0 * row_blocks) + in;
  BlockOf r;
  r.row = row0 + local / (unsigned)row_blocks;
  r.b = (int)(local % (unsigned)row_blocks);
  r.part = threadIdx.x & 3;
  r.in = base + in < blocks;
  return r;
}

// 1,000,003 x 400 fp32: 362 to 390 us, 1.82 GB at 4.7 to 5.0 TB/s, a large copy's rate; 10,000 x 50: 2.6 to 3 us, a launch.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_quantise(QuantiseArgs a) {
  typedef typename RowType<TYPE>::T T;
  const BlockOf at = block_of(a.first, a.blocks, a.row_blocks);
  if (!at.in) return;                                      // the four threads of a block go together
  float v[8];
  load8<TYPE>((const T*)a.x + at.row * a.x_stride, 32 * at.b + 8 * at.part, a.dim, v);
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  m = max(m, (unsigned)__shfl_xor((int)m, 1));
  m = max(m, (unsigned)__shfl_xor((int)m, 2));
  const bool finite = m < 0x7f800000u;
  const int scale = max((int)(m >> 23) - 2, 0);
  const float up = __uint_as_float((unsigned)(254 - scale) << 23);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= up;
  const unsigned codes = finite ? mx_codes(v) : 0u;
  *reinterpret_cast<unsigned*>(a.codes + at.row * a.codes_stride + 16 * at.b + 4 * at.part) = codes;
  if (at.part == 0) a.scales[at.row * a.scales_stride + at.b] = (uint8_t)(finite ? scale : 255);
}

struct RowsArgs {
  const uint8_t *codes, *scales; const int32_t* ids; void* out;
  int64_t codes_stride, scales_stride, out_stride, num_rows, blocks, first;
  int32_t dim, row_blocks;
};
// value = level (a conversion instruction's, exact) times 2^e.  1,000,003 x 400 to bf16: 227 to 250 us, 1.02 GB at 4.1 to 4.5 TB/s; 100,000
// rows by id out of 2,000,000: 19 us, 5.3 TB/s; 1,000 of 50 columns: 2.6 to 3 us, a launch.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_mxfp_rows(RowsArgs a) {
  typedef typename RowType<TYPE>::T T;
  const BlockOf at = block_of(a.first, a.blocks, a.row_blocks);
  if (!at.in) return;
  const int64_t id = a.ids ? a.ids[at.row] : at.row;
  unsigned codes = 0;
  float scale = 0.f;
  if (id >= 0 && id < a.num_rows) {
    codes = *reinterpret_cast<const unsigned*>(a.codes + id * a.codes_stride + 16 * at.b + 4 * at.part);
    scale = mx_scale(a.scales[id * a.scales_stride + at.b]);
  }
  float v[8];
  mx_values(codes, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= scale;
  const int c = 32 * at.b + 8 * at.part;
  if (c < a.dim) store8<TYPE>((T*)a.out + at.row * a.out_stride, c, a.dim, v);
}

// ------------------------------------------------------------------------------------------ entry points -----
static bool mxfp_dim_ok(int32_t dim) {
  if (dim >= 1 && dim <= MAR_MXFP_MAX_COLUMNS) return true;
  mar_set_error("dim outside 1..MAR_MXFP_MAX_COLUMNS");
  return false;
}

extern "C" int mar_mxfp_quantise(const void* x, int64_t x_stride, int64_t rows, int32_t dim, int32_t dtype, uint8_t* codes, int64_t codes_stride,
                                 uint8_t* scales, int64_t scales_stride, void* hip_stream) {
  if (dtype < MAR_DTYPE_FP32 || dtype > MAR_DTYPE_FP16) { mar_set_error("unknown dtype %d", dtype); return MAR_EINVAL; }
  if (rows < 0 || rows > 0x7fffffff) { mar_set_error("rows outside 0..2^31 - 1"); return MAR_ERANGE; }
  if (!mxfp_dim_ok(dim)) return MAR_ERANGE;
  if (x_stride < dim || x_stride > (int64_t)1 << 40) { mar_set_error("x_stride is below dim or above 2^40"); return MAR_EINVAL; }
  if (const char* why = mx_check_strides(dim, codes_stride, scales_stride)) { mar_set_error("%s", why); return MAR_EINVAL; }
  if (rows == 0) return MAR_OK;
  if (!x || !codes || !scales) { mar_set_error("x, codes or scales is NULL"); return MAR_EINVAL; }
  if ((uintptr_t)x & (dtype == MAR_DTYPE_FP32 ? 3 : 1)) { mar_set_error("x is not aligned to its type"); return MAR_EINVAL; }
  if ((uintptr_t)codes & 15) { mar_set_error("codes is not 16-byte aligned"); return MAR_EINVAL; }
  QuantiseArgs a;
  a.x = x; a.codes = codes; a.scales = scales;
  a.x_stride = x_stride; a.codes_stride = codes_stride; a.scales_stride = scales_stride;
  a.dim = dim; a.row_blocks = mx_blocks(dim); a.blocks = rows * a.row_blocks;
  const hipStream_t st = (hipStream_t)hip_stream;
  sm_launches((a.blocks + 63) / 64, 256, [&](int64_t first, unsigned blocks) {
    a.first = first;
    if (dtype == MAR_DTYPE_FP32) hipLaunchKernelGGL(k_quantise<0>, dim3(blocks), dim3(256), 0, st, a);
    else if (dtype == MAR_DTYPE_BF16) hipLaunchKernelGGL(k_quantise<1>, dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_quantise<2>, dim3(blocks), dim3(256), 0, st, a);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("quantisation kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}

extern "C" int mar_mxfp_rows(const uint8_t* codes, int64_t codes_stride, const uint8_t* scales, int64_t scales_stride, int64_t num_rows, int32_t dim,
                             const int32_t* ids, int64_t n, int32_t dtype, void* out, int64_t out_stride, void* hip_stream) {
  if (dtype < MAR_DTYPE_FP32 || dtype > MAR_DTYPE_FP16) { mar_set_error("unknown dtype %d", dtype); return MAR_EINVAL; }
  if (num_rows < 0 || num_rows > 0x7fffffff) { mar_set_error("num_rows outside 0..2^31 - 1"); return MAR_ERANGE; }
  if (n < 0 || n > 0x7fffffff) { mar_set_error("n outside 0..2^31 - 1"); return MAR_ERANGE; }
  if (!mxfp_dim_ok(dim)) return MAR_ERANGE;
  if (out_stride < dim || out_stride > (int64_t)1 << 40) { mar_set_error("out_stride is below dim or above 2^40"); return MAR_EINVAL; }
  if (const char* why = mx_check_strides(dim, codes_stride, scales_stride)) { mar_set_error("%s", why); return MAR_EINVAL; }
  if (n == 0) return MAR_OK;
  if (!out || (num_rows > 0 && (!codes || !scales))) { mar_set_error("codes, scales or out is NULL"); return MAR_EINVAL; }
  if ((uintptr_t)out & (dtype == MAR_DTYPE_FP32 ? 3 : 1)) { mar_set_error("out is not aligned to its type"); return MAR_EINVAL; }
  if ((uintptr_t)codes & 15) { mar_set_error("codes is not 16-byte aligned"); return MAR_EINVAL; }
  if ((uintptr_t)ids & 3) { mar_set_error("ids is not 4-byte aligned"); return MAR_EINVAL; }
  RowsArgs a;
  a.codes = codes; a.scales = scales; a.ids = ids; a.out = out;
  a.codes_stride = codes_stride; a.scales_stride = scales_stride; a.out_stride = out_stride; a.num_rows = num_rows;
  a.dim = dim; a.row_blocks = mx_blocks(dim); a.blocks = n * a.row_blocks;
  const hipStream_t st = (hipStream_t)hip_stream;
  sm_launches((a.blocks + 63) / 64, 256, [&](int64_t first, unsigned blocks) {
    a.first = first;
    if (dtype == MAR_DTYPE_FP32) hipLaunchKernelGGL(k_mxfp_rows<0>, dim3(blocks), dim3(256), 0, st, a);
    else if (dtype == MAR_DTYPE_BF16) hipLaunchKernelGGL(k_mxfp_rows<1>, dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_mxfp_rows<2>, dim3(blocks), dim3(256), 0, st, a);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("rows kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
