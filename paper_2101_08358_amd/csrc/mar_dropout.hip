// Dropout from the library's counter-based generator (gfx950): the mask is drawn again wherever it is needed and never stored.
//
// Eight columns 8 g .. 8 g + 7 of row r at step n share one block of Philox4x32-10: key = seed, counter = (r, g, n lo,
// 0xC0000000 | n hi), which no other draw of the library uses (sampling: top bit 0; table fill: 0x80000000 | table).  Column
// 8 g + e takes the lower (e even) or upper half u of output word e / 2 and is kept where u >= threshold = round(65536 p); a kept
// value is multiplied by 65536 / (65536 - threshold), so that its expectation is the value itself whatever p is rounded to.
//
// Sixteen bits a value halve the generator's work, twenty 32 x 32-bit products a block, and leave memory the bound: 100,000 x 400 fp32
// values 59 us (5.4 TB/s read and written), 16,001 x 4,096 bf16 42 us (6.2 TB/s); 1,000 x 50 3 us.
#include "mar_common.h"
#include "mar_philox.h"
#include "mar_rows_dev.h"

struct DropoutArgs {
  const void* x; void* out;
  int64_t x_stride, out_stride, rows, first;
  int32_t dim, groups;             // groups of eight columns to a row
  uint32_t threshold, k0, k1, n_lo, n_hi;
  float scale;
};

// A thread per group, from group `first` on.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_dropout(DropoutArgs a) {
  typedef typename RowType<TYPE>::T T;
  const int64_t at = a.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= a.rows * a.groups) return;
  const int64_t row = at / a.groups;
  const int g = (int)(at - row * a.groups);
  uint32_t c0 = (uint32_t)row, c1 = (uint32_t)g, c2 = a.n_lo, c3 = 0xC0000000u | a.n_hi;
  philox4x32_10(c0, c1, c2, c3, a.k0, a.k1);
  const uint32_t w[4] = {c0, c1, c2, c3};
  const T* x = (const T*)a.x + row * a.x_stride;
  T* out = (T*)a.out + row * a.out_stride;
  float v[8];
  load8<TYPE>(x, 8 * g, a.dim, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    v[e] = u >= a.threshold ? v[e] * a.scale : 0.f;
  }
  store8<TYPE>(out, 8 * g, a.dim, v);
}
#define DROPOUT_MAX_BLOCKS ((int64_t)1 << 23)               // a launch holds fewer than 2^32 threads (a loop in place of more launches: bf16 42 -> 50 us)

extern "C" int mar_dropout(const void* x, int64_t x_stride, int64_t rows, int32_t dim, int32_t dtype, float p, uint64_t seed,
                           uint64_t step, void* out, int64_t out_stride, void* hip_stream) {
  if (dtype < MAR_DTYPE_FP32 || dtype > MAR_DTYPE_FP16) { mar_set_error("unknown dtype %d", dtype); return MAR_EINVAL; }
  if (rows < 0 || rows > 0x7fffffff || dim < 1) { mar_set_error("rows outside 0..2^31 - 1 or dim below 1"); return MAR_ERANGE; }
  if (!(p >= 0.f && p < 1.f)) { mar_set_error("p must lie in [0, 1)"); return MAR_EINVAL; }
  const uint32_t threshold = (uint32_t)((double)p * 65536.0 + 0.5);
  if (threshold > 65535u) { mar_set_error("p is rounded to a multiple of 2^-16: at most 65535 / 65536"); return MAR_ERANGE; }
  if (step >> 62) { mar_set_error("step must be below 2^62"); return MAR_ERANGE; }
  if (x_stride < dim || out_stride < dim || x_stride > (int64_t)1 << 40 || out_stride > (int64_t)1 << 40) {
    mar_set_error("a stride is below dim or above 2^40"); return MAR_EINVAL;
  }
  if (rows == 0) return MAR_OK;
  if (!x || !out) { mar_set_error("x or out is NULL"); return MAR_EINVAL; }
  const uintptr_t align = dtype == MAR_DTYPE_FP32 ? 3 : 1;
  if (((uintptr_t)x & align) || ((uintptr_t)out & align)) { mar_set_error("x or out is not aligned to its type"); return MAR_EINVAL; }
  DropoutArgs a;
  a.x = x; a.out = out; a.x_stride = x_stride; a.out_stride = out_stride; a.rows = rows;
  a.dim = dim; a.groups = dim / 8 + (dim % 8 != 0);
  a.threshold = threshold; a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
  a.n_lo = (uint32_t)step; a.n_hi = (uint32_t)(step >> 32);
  a.scale = 65536.f / (float)(65536u - threshold);
  const int64_t blocks = (rows * a.groups + 255) / 256;
  if (blocks > 0x7fffffff) { mar_set_error("rows x dim is too large"); return MAR_ERANGE; }
  const hipStream_t st = (hipStream_t)hip_stream;
  for (int64_t b0 = 0; b0 < blocks; b0 += DROPOUT_MAX_BLOCKS) {
    const dim3 grid((unsigned)(blocks - b0 < DROPOUT_MAX_BLOCKS ? blocks - b0 : DROPOUT_MAX_BLOCKS));
    a.first = b0 * 256;
    if (dtype == MAR_DTYPE_FP32) hipLaunchKernelGGL(k_dropout<0>, grid, dim3(256), 0, st, a);
    else if (dtype == MAR_DTYPE_BF16) hipLaunchKernelGGL(k_dropout<1>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_dropout<2>, grid, dim3(256), 0, st, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("dropout kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
