// Scores of queries against every row of a table in microscaled 4-bit floats, on the matrix pipe's scaled 4- and 6-bit forms (gfx950).
//
// s_ij = scale sum_b 2^(e_jb) sum_(k in b) q_ik c_jk over blocks b of 32 columns.  The table enters the products as it lies: one lane's
// 32 columns of v_mfma_scale_f32_32x32x64 are one block with its own scale.  A query in 4 bits does likewise.  Other queries are written
// block by block as slices of signed base-32 digits,  q = sum_s d_s 2^(e - 3 - 5 s),  e the exponent of the block's largest magnitude,
// |d| <= 16:  d_s / 8 is a 6-bit float (2 exponent, 3 mantissa bits) whose code is |d| with the sign, 2^(e - 5 s) its block's scale.
// Five slices hold 24 bits of fp32 values, four 19 bits of 16-bit ones, counted from the block's largest value: every product is exact,
// sums are the matrix pipe's in fp32, smallest slice first.  6- and 4-bit operands run at four times the rate of 16-bit ones, so that five
// slices cost less than two 16-bit products, and the table takes a quarter of the registers that it would take in 16 bits.
//
// Lane layouts (lane = 32 h + m): A lane holds query m, block 2 k + h of step k; B lane the same block of table row m; D lane holds
// row m, register r = query 8 (r / 4) + 4 h + r % 4.
#include "mar_common.h"
#include "mar_mxfp.h"
#include "mar_rows_dev.h"
#include "mar_softmax.h"

typedef int mx_v8 __attribute__((ext_vector_type(8)));
typedef float mx_f16 __attribute__((ext_vector_type(16)));

// Images of 32 queries each: [slice][step]: 16 bytes of every lane, then (6-bit slices) 8 more; then the scales of every slice, a byte a step.
template <int NK, int NS> struct MxImage {
  static constexpr int FRAG = NS == 1 ? 1024 : 1536, NW = (NK + 3) / 4;
  static constexpr int SCALES = NS * NK * FRAG, BYTES = SCALES + NS * NW * 256;
};
static int mx_image_bytes(int nk, int ns) { return ns * nk * (ns == 1 ? 1024 : 1536) + ns * ((nk + 3) / 4) * 256; }

struct MxArgs {
  const void* queries; const uint8_t* query_scales;
  const uint8_t *codes, *scales;
  void* out; char* images;
  int64_t query_stride, query_scales_stride, codes_stride, scales_stride, out_stride;
  int32_t n, num_rows, dim, row_blocks, out_type;
  int32_t stripes, parts, tiles_part;    // stripes of rows; parts of the queries' tiles, tiles each
  float scale;
};

// A thread per lane of a step's operand.
template <int TYPE, int NK, int NS>
__global__ void __launch_bounds__(256)
k_mxfp_pack(MxArgs a) {
  typedef MxImage<NK, NS> I;
  const int lane = threadIdx.x & 63, unit = (int)blockIdx.x * 4 + (threadIdx.x >> 6), tile = unit / NK, k = unit - tile * NK;
  const int64_t q = (int64_t)tile * 32 + (lane & 31);
  if ((int64_t)tile * 32 >= a.n) return;
  const int b = 2 * k + (lane >> 5);
  const bool in = q < a.n && b < a.row_blocks;
  char* image = a.images + (size_t)tile * I::BYTES;
  uint8_t* scales = (uint8_t*)image + I::SCALES + ((k / 4) * 64 + lane) * 4 + k % 4;
  if constexpr (TYPE == 3) {
    row_u4 c = {0u, 0u, 0u, 0u};
    if (in) c = *reinterpret_cast<const row_u4*>((const uint8_t*)a.queries + q * a.query_stride + 16 * b);
    *reinterpret_cast<row_u4*>(image + k * 1024 + lane * 16) = c;
    *scales = in ? a.query_scales[q * a.query_scales_stride + b] : (uint8_t)127;
  } else {
    typedef typename RowType<TYPE>::T T;
    float v[32];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float part[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (in) load8<TYPE>((const T*)a.queries + q * a.query_stride, 32 * b + 8 * j, a.dim, part);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[8 * j + e] = part[e];
    }
    unsigned largest = 0;
#pragma unroll
    for (int e = 0; e < 32; ++e) largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
    const bool finite = largest < 0x7f800000u;
    const int field = max((int)(largest >> 23), 1);        // e + 127
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = finite ? __builtin_ldexpf(v[e], 130 - field) : 0.f;   // largest in [8, 16)
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      unsigned w[6] = {0u, 0u, 0u, 0u, 0u, 0u};
      const bool held = field - 5 * s >= 0;                // scales end at 2^-127
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float d = rintf(v[e]);
        v[e] = (v[e] - d) * 32.f;
        const unsigned c = (unsigned)fabsf(d) | (__float_as_uint(d) >> 31) << 5;
        const int at = 6 * e;
        w[at / 32] |= c << (at % 32);
        if (at % 32 > 26) w[at / 32 + 1] |= c >> (32 - at % 32);
      }
      char* frag = image + (s * NK + k) * I::FRAG;
      row_u4 lo = {w[0], w[1], w[2], w[3]};
      uint2 hi = make_uint2(w[4], w[5]);
      if (!held) { lo = (row_u4)(0u); hi = make_uint2(0u, 0u); }
      *reinterpret_cast<row_u4*>(frag + lane * 16) = lo;
      *reinterpret_cast<uint2*>(frag + 1024 + lane * 8) = hi;
      scales[s * I::NW * 256] = (uint8_t)(finite ? max(field - 5 * s, 0) : 255);
    }
  }
}

// One slice's products with RT x 32 rows: step K's scales are byte K % 4 of their words.
template <int K, int NK, int NS, int RT>
__device__ __forceinline__ void mx_steps(const char* frags, int lane, const int* qs, const row_u4 (&w)[RT][NK], const int (&ws)[RT][(NK + 3) / 4], mx_f16 (&acc)[RT]) {
  if constexpr (K < NK) {
    typedef MxImage<NK, NS> I;
    mx_v8 q = {0, 0, 0, 0, 0, 0, 0, 0};
    const row_u4 lo = *reinterpret_cast<const row_u4*>(frags + K * I::FRAG + lane * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = (int)lo[i];
    if constexpr (NS > 1) {
      const uint2 hi = *reinterpret_cast<const uint2*>(frags + K * I::FRAG + 1024 + lane * 8);
      q[4] = (int)hi.x; q[5] = (int)hi.y;
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const mx_v8 r = {(int)w[t][K][0], (int)w[t][K][1], (int)w[t][K][2], (int)w[t][K][3], 0, 0, 0, 0};
      // operand types: 2 = 6 bits (2 exponent, 3 mantissa), 4 = 4 bits
      acc[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(q, r, acc[t], NS > 1 ? 2 : 4, 4, K % 4, qs[K / 4], K % 4, ws[t][K / 4]);
    }
    mx_steps<K + 1, NK, NS, RT>(frags, lane, qs, w, ws, acc);
  }
}

// A wave holds 32 RT rows of the table in registers, lane m's RT rows neighbours, and takes the queries' images one by one out of LDS.
template <int NK, int NS, int RT>
__global__ void __launch_bounds__(256)
k_mxfp_scores(MxArgs a) {
  typedef MxImage<NK, NS> I;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 31, h = lane >> 5;
  const int part = (int)blockIdx.x / a.stripes, stripe = (int)blockIdx.x - part * a.stripes;
  const int row0 = (stripe * 4 + wave) * 32 * RT + m * RT;
  const int tiles = (a.n + 31) / 32, t0 = part * a.tiles_part, t1 = min(tiles, t0 + a.tiles_part);

  row_u4 w[RT][NK];
  int ws[RT][I::NW];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t row = min(row0 + t, a.num_rows - 1);     // rows beyond the last are taken and not written
    const uint8_t* codes = a.codes + row * a.codes_stride;
    const uint8_t* scales = a.scales + row * a.scales_stride;
#pragma unroll
    for (int k = 0; k < I::NW; ++k) ws[t][k] = 0;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int b = 2 * k + h;
      w[t][k] = (row_u4)(0u);
      unsigned s = 0;
      if (b < a.row_blocks) { w[t][k] = *reinterpret_cast<const row_u4*>(codes + 16 * b); s = scales[b]; }
      ws[t][k / 4] |= s << (8 * (k % 4));
    }
  }
  for (int tile = t0; tile < t1; ++tile) {
    __syncthreads();
    const char* image = a.images + (size_t)tile * I::BYTES;
    for (int at = tid * 16; at < I::BYTES; at += 256 * 16) *reinterpret_cast<row_u4*>(smem + at) = *reinterpret_cast<const row_u4*>(image + at);
    __syncthreads();
    mx_f16 acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = (mx_f16)(0.f);
#pragma unroll
    for (int s = NS - 1; s >= 0; --s) {
      int qs[I::NW];
#pragma unroll
      for (int k = 0; k < I::NW; ++k) qs[k] = *reinterpret_cast<const int*>(smem + I::SCALES + ((s * I::NW + k) * 64 + lane) * 4);
      mx_steps<0, NK, NS, RT>(smem + s * NK * I::FRAG, lane, qs, w, ws, acc);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t q = (int64_t)tile * 32 + 8 * (r / 4) + 4 * h + r % 4;
      float v[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) v[t] = acc[t][r] * a.scale;
      if (q < a.n) {
        if (a.out_type == 0) store_cols<0, RT>((float*)a.out + q * a.out_stride, row0, a.num_rows, v);
        else if (a.out_type == 1) store_cols<1, RT>((__bf16*)a.out + q * a.out_stride, row0, a.num_rows, v);
        else store_cols<2, RT>((_Float16*)a.out + q * a.out_stride, row0, a.num_rows, v);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------ launches -----
static int mx_slices(int dtype) { return dtype == MAR_DTYPE_MXFP4 ? 1 : (dtype == MAR_DTYPE_FP32 ? 5 : 4); }
static int64_t mx_tiles(int64_t queries) { return (queries + 31) / 32; }

struct MxPlan { int rt, stripes, parts, tiles_part; };
static MxPlan mx_plan(const mar_mxfp* p) {
  MxPlan r;
  const int64_t tiles = mx_tiles(p->num_queries);
  r.rt = p->num_rows * tiles >= 4 * 32 * 1024 ? 4 : 1;
  r.stripes = (int)((p->num_rows + 128 * r.rt - 1) / (128 * r.rt));
  int64_t parts = (1024 + r.stripes - 1) / r.stripes;
  if (parts > tiles) parts = tiles;
  r.tiles_part = (int)((tiles + parts - 1) / parts);
  r.parts = (int)((tiles + r.tiles_part - 1) / r.tiles_part);
  return r;
}

template <int TYPE, int NK> static void launch_pack(const MxArgs& a, hipStream_t st) {
  constexpr int NS = TYPE == 3 ? 1 : (TYPE == 0 ? 5 : 4);
  const int64_t units = mx_tiles(a.n) * NK;
  hipLaunchKernelGGL((k_mxfp_pack<TYPE, NK, NS>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st, a);
}
template <int NK> static void launch_nk(int dtype, int rt, const MxArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_pack<0, NK>(a, st); else if (dtype == MAR_DTYPE_BF16) launch_pack<1, NK>(a, st);
  else if (dtype == MAR_DTYPE_FP16) launch_pack<2, NK>(a, st); else launch_pack<3, NK>(a, st);
  const dim3 grid((unsigned)(a.stripes * a.parts)), block(256);
  const int ns = mx_slices(dtype);
  if (rt == 4) {
    if (ns == 5) hipLaunchKernelGGL((k_mxfp_scores<NK, 5, 4>), grid, block, (MxImage<NK, 5>::BYTES), st, a);
    else if (ns == 4) hipLaunchKernelGGL((k_mxfp_scores<NK, 4, 4>), grid, block, (MxImage<NK, 4>::BYTES), st, a);
    else hipLaunchKernelGGL((k_mxfp_scores<NK, 1, 4>), grid, block, (MxImage<NK, 1>::BYTES), st, a);
  } else {
    if (ns == 5) hipLaunchKernelGGL((k_mxfp_scores<NK, 5, 1>), grid, block, (MxImage<NK, 5>::BYTES), st, a);
    else if (ns == 4) hipLaunchKernelGGL((k_mxfp_scores<NK, 4, 1>), grid, block, (MxImage<NK, 4>::BYTES), st, a);
    else hipLaunchKernelGGL((k_mxfp_scores<NK, 1, 1>), grid, block, (MxImage<NK, 1>::BYTES), st, a);
  }
}

// ------------------------------------------------------------------------------------------ entry points -----
static const char* mx_check(const mar_mxfp* p, int* code) {
  *code = MAR_EINVAL;
  if (!p) return "problem is NULL";
  if (p->reserved != 0) return "reserved must be 0";
  if (p->dtype < MAR_DTYPE_FP32 || p->dtype > MAR_DTYPE_MXFP4) return "unknown dtype";
  if (p->score_dtype < MAR_DTYPE_FP32 || p->score_dtype > MAR_DTYPE_FP16) return "unknown score_dtype";
  if (!(p->scale >= 1e-6f && p->scale <= 1e6f)) return "scale outside 1e-6 .. 1e6";
  *code = MAR_ERANGE;
  if (p->num_rows < 1 || p->num_rows > MAR_SOFTMAX_MAX_ROWS) return "num_rows outside 1..MAR_SOFTMAX_MAX_ROWS";
  if (p->num_queries < 0 || p->num_queries > MAR_SOFTMAX_MAX_QUERIES) return "num_queries outside 0..MAR_SOFTMAX_MAX_QUERIES";
  if (p->dim < 1 || p->dim > MAR_MAX_DIM) return "dim outside 1..MAR_MAX_DIM";
  *code = MAR_EINVAL;
  if (const char* why = mx_check_strides(p->dim, p->codes_stride, p->scales_stride)) return why;
  if (p->dtype == MAR_DTYPE_MXFP4) {
    if (mx_check_strides(p->dim, p->query_stride, p->query_scales_stride)) return "a stride of the queries' codes or scales does not fit";
  } else if (p->query_stride < p->dim || p->query_stride > (int64_t)1 << 40) return "query_stride is below dim or above 2^40";
  if (p->score_stride < p->num_rows || p->score_stride > (int64_t)1 << 40) return "score_stride is below num_rows or above 2^40";
  return nullptr;
}

extern "C" int mar_mxfp_scores_workspace_bytes(const mar_mxfp* p, size_t* out_bytes) {
  int code;
  if (const char* why = mx_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (!out_bytes) { mar_set_error("out_bytes is NULL"); return MAR_EINVAL; }
  const size_t bytes = (size_t)mx_tiles(p->num_queries) * mx_image_bytes((p->dim + 63) / 64, mx_slices(p->dtype));
  *out_bytes = bytes > 256 ? bytes : 256;
  return MAR_OK;
}

extern "C" int mar_mxfp_scores(const mar_mxfp* p, const void* queries, const uint8_t* query_scales, const uint8_t* codes, const uint8_t* scales,
                               void* scores, void* workspace, size_t workspace_bytes, void* hip_stream) {
  size_t need;
  const int rc = mar_mxfp_scores_workspace_bytes(p, &need);
  if (rc != MAR_OK) return rc;
  const bool four = p->dtype == MAR_DTYPE_MXFP4;
  if (!codes || !scales) { mar_set_error("codes or scales is NULL"); return MAR_EINVAL; }
  if (p->num_queries > 0 && (!queries || !scores || (four && !query_scales))) { mar_set_error("queries, query_scales or scores is NULL"); return MAR_EINVAL; }
  if (((uintptr_t)codes & 15) || (four && ((uintptr_t)queries & 15))) { mar_set_error("codes are not 16-byte aligned"); return MAR_EINVAL; }
  if ((!four && ((uintptr_t)queries & (p->dtype == MAR_DTYPE_FP32 ? 3 : 1))) || ((uintptr_t)scores & (p->score_dtype == MAR_DTYPE_FP32 ? 3 : 1))) {
    mar_set_error("a matrix is not aligned to its type"); return MAR_EINVAL;
  }
  if (!workspace || ((uintptr_t)workspace & 255)) { mar_set_error("workspace must be non-NULL and 256-byte aligned"); return MAR_EINVAL; }
  if (workspace_bytes < need) { mar_set_error("workspace has %zu bytes, %zu needed", workspace_bytes, need); return MAR_ENOMEM; }
  if (p->num_queries == 0) return MAR_OK;
  MxArgs a = {};
  const MxPlan plan = mx_plan(p);
  a.queries = queries; a.query_scales = query_scales; a.codes = codes; a.scales = scales; a.out = scores; a.images = (char*)workspace;
  a.query_stride = p->query_stride; a.query_scales_stride = p->query_scales_stride; a.codes_stride = p->codes_stride; a.scales_stride = p->scales_stride;
  a.out_stride = p->score_stride; a.n = p->num_queries; a.num_rows = (int32_t)p->num_rows; a.dim = p->dim; a.row_blocks = mx_blocks(p->dim);
  a.out_type = p->score_dtype; a.stripes = plan.stripes; a.parts = plan.parts; a.tiles_part = plan.tiles_part; a.scale = p->scale;
  const hipStream_t st = (hipStream_t)hip_stream;
  switch ((p->dim + 63) / 64) {
    case 1: launch_nk<1>(p->dtype, plan.rt, a, st); break;
    case 2: launch_nk<2>(p->dtype, plan.rt, a, st); break;
    case 3: launch_nk<3>(p->dtype, plan.rt, a, st); break;
    case 4: launch_nk<4>(p->dtype, plan.rt, a, st); break;
    case 5: launch_nk<5>(p->dtype, plan.rt, a, st); break;
    case 6: launch_nk<6>(p->dtype, plan.rt, a, st); break;
    default: launch_nk<7>(p->dtype, plan.rt, a, st); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("score kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
