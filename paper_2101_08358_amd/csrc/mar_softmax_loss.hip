// Softmax cross entropy over all rows of a table, with the gradients of queries and table (gfx950): pass 1 (statistics and the
// weighted sum of rows for every query), k_loss_rows (joins the parts: log-sum-exp, loss, the queries' gradient), pass 2 (the
// table's gradient, scores computed again), k_loss_table (adds its parts).
//
// 10,000 queries, 14,951 rows of 100 floats, us: layout 7, pass 1 208 (1,050 TFLOP/s of 16-bit products counting padded columns), k_loss_rows
// 23, pass 2 244, k_loss_table 6; 8,192 queries, 65,536 bf16 rows of 400 columns: 20, 900 to 970, 18, 1,050 to 1,100.  A large
// library product reaches 1,170 TFLOP/s on the card (1,190 to 1,240 on others), whose clock gives way to its power limit.
#include "mar_softmax_dev.h"

struct LossArgs {
  const void *Q, *W; int64_t q_stride, w_stride;
  int32_t n, dim, parts, o_pitch;
  int64_t rows;
  float scale; double unscale;     // natural units of a reference's: scale / c
  const int32_t* targets; const float* weights;
  const float4* stats; const float* O;
  float *row_m, *row_f, *row_u;
  float *loss, *lse;
  void* grad; int64_t grad_stride;
};

// WAVES waves per query: wave w takes parts w, w + WAVES, ..
template <int TYPE, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_loss_rows(LossArgs a) {
  typedef typename RowType<TYPE>::T T;
  __shared__ float fac[MAR_SOFTMAX_MAX_PARTS];
  __shared__ float4 sums[WAVES][(MAR_MAX_DIM + 3) / 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t q = blockIdx.x;
  // every wave for itself: a lane a part
  const float4 mine = lane < a.parts ? a.stats[(size_t)lane * a.n + q] : make_float4(SM_NO_REF, 0.f, SM_NO_REF, 0.f);
  float mo = mine.x, m = mine.z;                           // references of the sums of rows and of weights
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) { mo = fmaxf(mo, __shfl_xor(mo, o)); m = fmaxf(m, __shfl_xor(m, o)); }
  const float f = __builtin_amdgcn_exp2f(mine.x - mo);
  float l = mine.y * __builtin_amdgcn_exp2f(mine.z - m);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o);
  if (wave == 0) fac[lane] = f;
  const int t = a.targets[q];
  const bool has = t >= 0 && t < a.rows;
  const float given = has ? (a.weights ? a.weights[q] : 1.f) : 0.f;
  const float u = fabsf(given) < SM_LEAST_WEIGHT ? 0.f : given;
  const T* qr = (const T*)a.Q + q * a.q_stride;
  const T* wr = (const T*)a.W + (int64_t)(has ? t : 0) * a.w_stride;
  double dot = 0.0;
  for (int c = lane; c < a.dim; c += 64) dot = __builtin_fma((double)(float)qr[c], (double)(float)wr[c], dot);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) dot += __shfl_xor(dot, o);
  const double lse = (double)m * a.unscale + log_of_sum(l), over = at_most_0(dot * (double)a.scale - lse);   // log p of the answer
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[q] = (float)lse;
    if (a.loss) a.loss[q] = u != 0.f ? (float)(-(double)u * over) : 0.f;
    if (a.row_m) {
      // the integer and the logarithm of the mantissa stay apart: their sum would be rounded to 2^-19, the same for all of a query's weights
      int e = 0;
      const float mantissa = frexpf(l, &e);
      a.row_m[q] = u != 0.f ? m + (float)e : 0.f;
      a.row_u[q] = u;
      const float lu = log2f(fabsf(u));
      a.row_f[q] = u != 0.f ? lu - log2f(mantissa) : -__builtin_inff();
    }
  }
  if (!a.grad) return;
  __syncthreads();
  const int quads = a.o_pitch / 4;
  for (int c = lane; c < quads; c += 64) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* O = a.O + (size_t)q * a.o_pitch + 4 * c;
#pragma unroll 4
    for (int p = wave; p < a.parts; p += WAVES) {
      const float4 v = *reinterpret_cast<const float4*>(O + (size_t)p * a.n * a.o_pitch);
      const float k = fac[p];
      sum.x = __builtin_fmaf(v.x, k, sum.x); sum.y = __builtin_fmaf(v.y, k, sum.y); sum.z = __builtin_fmaf(v.z, k, sum.z); sum.w = __builtin_fmaf(v.w, k, sum.w);
    }
    sums[wave][c] = sum;
  }
  __syncthreads();
  T* out = (T*)a.grad + q * a.grad_stride;
  const float less = expm1f((float)over), inv = 1.f / l, us = u * a.scale;
  const int up = (int)(mo - m);
  for (int c = threadIdx.x; c < a.dim; c += 64 * WAVES) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += reinterpret_cast<const float*>(sums[w])[c];
    const float v = us * __builtin_fmaf(less, (float)wr[c], __builtin_ldexpf(sum * inv, up));
    out[c] = (T)(u != 0.f ? v : 0.f);
  }
}
template <int TYPE> static void launch_rows(const LossArgs& a, hipStream_t st) {
  if (sm_loss_waves(a.parts, a.n) == 4) hipLaunchKernelGGL((k_loss_rows<TYPE, 4>), dim3((unsigned)a.n), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_loss_rows<TYPE, 1>), dim3((unsigned)a.n), dim3(64), 0, st, a);
}

// Adds the parts of pass 2: a thread per four columns, from workgroup `begin` on.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_loss_table(const float* __restrict__ O, int parts, int64_t rows, int dim, int o_pitch, void* grad, int64_t stride, int64_t begin) {
  typedef typename RowType<TYPE>::T T;
  const int64_t at = (begin + blockIdx.x) * 256 + threadIdx.x;
  const int quads = o_pitch / 4;
  const int64_t row = at / quads;
  if (row >= rows) return;
  const int c = 4 * (int)(at - row * quads);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < parts; ++p) {
    const float4 o = *reinterpret_cast<const float4*>(O + ((size_t)p * rows + row) * o_pitch + c);
    v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
  }
  store_cols<TYPE, 4>((T*)grad + row * stride, c, dim, v);
}

// ------------------------------------------------------------------------------------------ launches -----
template <int TYPE, int PASS>
static void launch_nk(const SmArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.units + 7) / 8 * 8)), block(256);
  switch (sm_nk(a.dim)) {
    case 2: hipLaunchKernelGGL((k_softmax<TYPE, 2, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_softmax<TYPE, 4, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    case 7: hipLaunchKernelGGL((k_softmax<TYPE, 7, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((k_softmax<TYPE, 8, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    case 12: hipLaunchKernelGGL((k_softmax<TYPE, 12, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    case 16: hipLaunchKernelGGL((k_softmax<TYPE, 16, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_softmax<TYPE, 25, PASS, SM_IMAGES>), grid, block, 0, st, a); break;
  }
}
template <int PASS> static hipError_t launch_pass(int dtype, const SmArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_nk<0, PASS>(a, st);
  else if (dtype == MAR_DTYPE_BF16) launch_nk<1, PASS>(a, st);
  else launch_nk<2, PASS>(a, st);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------ entry points -----
// Workspace: images of both matrices, statistics, the queries' sums, what pass 2 reads per query, the parts of the table's gradient.
struct LossLayout { size_t qtiles, qexps, wtiles, wexps, stats, O1, row_m, row_f, row_u, O2, bytes; SmPlan p1, p2; int32_t o_pitch; };

static LossLayout loss_layout(const mar_softmax* p) {
  LossLayout L;
  L.p1 = sm_plan(p->dtype, p->dim, 1, SM_IMAGES, p->num_queries, p->num_rows, 1);
  L.p2 = sm_plan(p->dtype, p->dim, 2, SM_IMAGES, p->num_rows, p->num_queries, 1);
  L.o_pitch = (p->dim + 3) / 4 * 4;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  const size_t T = (size_t)p->num_queries;
  L.qtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_queries)); L.qexps = take(sm_exps_bytes(p->num_queries));
  L.wtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_rows)); L.wexps = take(sm_exps_bytes(p->num_rows));
  L.stats = take((size_t)L.p1.parts * T * sizeof(float4));
  L.O1 = take((size_t)L.p1.parts * T * L.o_pitch * 4);
  L.row_m = take(T * 4); L.row_f = take(T * 4); L.row_u = take(T * 4);
  L.O2 = take(L.p2.parts > 1 ? (size_t)L.p2.parts * p->num_rows * L.o_pitch * 4 : 0);
  L.bytes = at > 256 ? at : 256;
  return L;
}

extern "C" int mar_softmax_loss_workspace_bytes(const mar_softmax* p, size_t* out_bytes) {
  int code;
  if (const char* why = sm_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (!out_bytes) { mar_set_error("out_bytes is NULL"); return MAR_EINVAL; }
  *out_bytes = loss_layout(p).bytes;
  return MAR_OK;
}

extern "C" int mar_softmax_loss(const mar_softmax* p, const void* queries, const void* table, const int32_t* targets, const float* weights,
                                float* loss, float* lse, void* grad_queries, int64_t grad_query_stride, void* grad_table,
                                int64_t grad_row_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int code;
  if (const char* why = sm_check(p, &code)) { mar_set_error("%s", why); return code; }
  const uintptr_t align = p->dtype == MAR_DTYPE_FP32 ? 3 : 1;
  if (!table || (p->num_queries > 0 && (!queries || !targets))) { mar_set_error("queries, table or targets is NULL"); return MAR_EINVAL; }
  if (((uintptr_t)queries | (uintptr_t)table | (uintptr_t)grad_queries | (uintptr_t)grad_table) & align) { mar_set_error("a matrix is not aligned to its type"); return MAR_EINVAL; }
  if (((uintptr_t)targets | (uintptr_t)weights | (uintptr_t)loss | (uintptr_t)lse) & 3) { mar_set_error("an array is not 4-byte aligned"); return MAR_EINVAL; }
  if ((grad_queries && grad_query_stride < p->dim) || (grad_table && grad_row_stride < p->dim)) { mar_set_error("a gradient's stride is below dim"); return MAR_EINVAL; }
  if (!workspace || ((uintptr_t)workspace & 255)) { mar_set_error("workspace must be non-NULL and 256-byte aligned"); return MAR_EINVAL; }
  const LossLayout L = loss_layout(p);
  if (workspace_bytes < L.bytes) { mar_set_error("workspace has %zu bytes, %zu needed", workspace_bytes, L.bytes); return MAR_ENOMEM; }
  const hipStream_t st = (hipStream_t)hip_stream;
  char* const ws = (char*)workspace;
  const float c = p->scale * 1.44269504088896341f;

  SmArgs a = {};
  a.dim = p->dim; a.c = c; a.scale = p->scale; a.o_pitch = L.o_pitch; a.targets = targets; a.weights = weights;
  const SmImage qimg = sm_image(ws + L.qtiles, ws + L.qexps, p->num_queries), wimg = sm_image(ws + L.wtiles, ws + L.wexps, p->num_rows);
  SmPackArgs w = {}, k = {};
  w.dim = k.dim = p->dim;
  w.src = table; w.stride = p->row_stride; w.n = (int32_t)p->num_rows; w.to = wimg;
  k.src = queries; k.stride = p->query_stride; k.n = p->num_queries; k.to = qimg;
  k.ids = targets; k.weights = weights; k.num_ids = p->num_rows; k.least_weight = SM_LEAST_WEIGHT;
  hipError_t e = sm_pack(p->dtype, w, k, st);
  if (e != hipSuccess) { mar_set_error("image kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  if (p->num_queries > 0) {
    a.ximg = qimg; a.n_x = p->num_queries;
    a.yimg = wimg; a.n_y = (int32_t)p->num_rows;
    a.nstripes = L.p1.stripes; a.parts = L.p1.parts; a.tps = L.p1.tps; a.units = a.nstripes * a.parts;
    a.stats = (float4*)(ws + L.stats); a.O = (float*)(ws + L.O1);
    e = launch_pass<1>(p->dtype, a, st);
    if (e != hipSuccess) { mar_set_error("softmax kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
    LossArgs r = {};
    r.Q = queries; r.W = table; r.q_stride = p->query_stride; r.w_stride = p->row_stride;
    r.n = p->num_queries; r.dim = p->dim; r.parts = L.p1.parts; r.o_pitch = L.o_pitch; r.rows = p->num_rows;
    r.scale = p->scale; r.unscale = (double)p->scale / (double)c;
    r.targets = targets; r.weights = weights; r.stats = a.stats; r.O = a.O;
    if (grad_table) { r.row_m = (float*)(ws + L.row_m); r.row_f = (float*)(ws + L.row_f); r.row_u = (float*)(ws + L.row_u); }
    r.loss = loss; r.lse = lse; r.grad = grad_queries; r.grad_stride = grad_query_stride;
    if (p->dtype == MAR_DTYPE_FP32) launch_rows<0>(r, st); else if (p->dtype == MAR_DTYPE_BF16) launch_rows<1>(r, st); else launch_rows<2>(r, st);
    e = hipGetLastError();
    if (e != hipSuccess) { mar_set_error("loss kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  }
  if (!grad_table) return MAR_OK;
  a.ximg = wimg; a.n_x = (int32_t)p->num_rows;
  a.yimg = qimg; a.n_y = p->num_queries;
  a.nstripes = L.p2.stripes; a.parts = L.p2.parts; a.tps = L.p2.tps; a.units = a.nstripes * a.parts;
  a.row_m = (const float*)(ws + L.row_m); a.row_f = (const float*)(ws + L.row_f); a.row_u = (const float*)(ws + L.row_u);
  a.O = (float*)(ws + L.O2);
  if (L.p2.parts == 1) { a.out = grad_table; a.out_stride = grad_row_stride; }
  e = launch_pass<2>(p->dtype, a, st);
  if (e == hipSuccess && L.p2.parts > 1) {
    sm_launches((p->num_rows * (L.o_pitch / 4) + 255) / 256, 256, [&](int64_t first, unsigned blocks) {
      const dim3 grid(blocks), block(256);
      if (p->dtype == MAR_DTYPE_FP32) hipLaunchKernelGGL(k_loss_table<0>, grid, block, 0, st, a.O, L.p2.parts, p->num_rows, p->dim, L.o_pitch, grad_table, grad_row_stride, first);
      else if (p->dtype == MAR_DTYPE_BF16) hipLaunchKernelGGL(k_loss_table<1>, grid, block, 0, st, a.O, L.p2.parts, p->num_rows, p->dim, L.o_pitch, grad_table, grad_row_stride, first);
      else hipLaunchKernelGGL(k_loss_table<2>, grid, block, 0, st, a.O, L.p2.parts, p->num_rows, p->dim, L.o_pitch, grad_table, grad_row_stride, first);
    });
    e = hipGetLastError();
  }
  if (e != hipSuccess) { mar_set_error("table gradient kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
