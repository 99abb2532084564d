// Log probabilities over all rows of a table: of given answers, with the distribution's entropy and its most probable rows (gfx950).
//
// Pass 0 (mar_softmax_dev.h) leaves statistics per query and part of the table, and the largest score of every group of 16
// group_tiles rows.  k_answer joins the parts, a workgroup per query; the most probable rows lie in the groups with the largest
// maxima, whose rows are scored again: in fp32, and the best of them in 64 bits, by which they are ordered.
#include "mar_softmax_dev.h"

// Stripes of queries from which the table is laid out as images first.
#ifndef MAR_SOFTMAX_IMAGES
#define MAR_SOFTMAX_IMAGES 8
#endif
#define SM_MARGIN 4               // groups, and rows, kept beyond the number asked for: what fp32 cannot tell apart

struct AnswerArgs {
  const void *Q, *W; int64_t q_stride, w_stride, rows;
  int32_t n, dim, parts, num_top, group_tiles;
  int64_t ngroups;                 // 0: no group maxima
  float scale; double unscale;
  const int32_t* targets;
  const uint32_t* allowed; int64_t allowed_stride;
  const float4* stats; const float* gmax;
  float *log_probs, *entropy, *top_log_probs; int32_t* top_ids;
};

// Ascending with the value: -inf, NaN: 0, never chosen.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v);
  if (!(v > -__builtin_inff())) return 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The `want` largest of keys[0 .. n) (all different, 0: none), in descending order in best[]; returns how many there are.
// A threshold with at least `want` and at most `CAP` keys above it is found by bisection, those keys are ranked.
template <int NT, int CAP>
__device__ int select_top(const unsigned long long* keys, int n, int want, unsigned long long* cand, unsigned long long* best, int* cnt) {
  const int tid = threadIdx.x;
  auto count = [&](unsigned long long x, int turn) {
    int c = 0;
    for (int e = tid; e < n; e += NT) c += keys[e] >= x ? 1 : 0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) c += __shfl_xor(c, o);
    if ((tid & 63) == 0) cnt[(turn & 1) * (NT / 64) + (tid >> 6)] = c;
    __syncthreads();
    c = 0;
    for (int w = 0; w < NT / 64; ++w) c += cnt[(turn & 1) * (NT / 64) + w];
    return c;
  };
  __syncthreads();                                         // the keys are written
  unsigned long long lo = 1, hi = ~0ull;
  int turn = 0, c = count(lo, turn++);
  unsigned long long x = lo;
  if (c > CAP) {
    while (hi - lo > 1) {                                  // at least `lo`: more than CAP keys, at least `hi`: fewer than `want`
      x = lo + (hi - lo) / 2;
      c = count(x, turn++);
      if (c > CAP) lo = x; else if (c < want) hi = x; else break;
    }
  }
  __syncthreads();
  if (tid == 0) cnt[0] = 0;
  __syncthreads();
  for (int e = tid; e < n; e += NT) {
    if (keys[e] >= x) { const int at = atomicAdd(&cnt[0], 1); if (at < CAP) cand[at] = keys[e]; }
  }
  __syncthreads();
  const int have = min(cnt[0], CAP);
  for (int e = tid; e < have; e += NT) {
    const unsigned long long k = cand[e];
    int rank = 0;
    for (int j = 0; j < have; ++j) rank += cand[j] > k ? 1 : 0;
    if (rank < want) best[rank] = k;
  }
  __syncthreads();
  return min(have, want);
}

// CHUNK: keys looked at together; best ones are carried from chunk to chunk.
template <int TYPE, int NT, int CHUNK>
__global__ void __launch_bounds__(NT)
k_answer(AnswerArgs a) {
  typedef typename RowType<TYPE>::T T;
  constexpr int CAP = 128, MAXW = MAR_MAX_TOP + SM_MARGIN;
  __shared__ float s_m[NT / 64], s_l[NT / 64], s_a[NT / 64];
  __shared__ float qs[512];
  __shared__ unsigned long long keys[CHUNK + MAXW], cand[CAP], best[MAXW];
  __shared__ double exact[MAXW];
  __shared__ int cnt[2 * (NT / 64)], groups[MAXW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t q = blockIdx.x;
  const T* qr = (const T*)a.Q + q * a.q_stride;
  const T* W = (const T*)a.W;
  const uint32_t* allowed = a.allowed ? a.allowed + q * a.allowed_stride : nullptr;
  auto is_allowed = [&](int64_t row) { return !allowed || (allowed[row >> 5] >> (row & 31) & 1u); };

  // ---- statistics of all parts
  auto join = [](float& m, float& l, float& s, float m2, float l2, float s2) {
    const float to = fmaxf(m, m2), d1 = m - to, d2 = m2 - to, f1 = __builtin_amdgcn_exp2f(d1), f2 = __builtin_amdgcn_exp2f(d2);
    const float sa = l != 0.f ? f1 * __builtin_fmaf(d1, l, s) : 0.f, sb = l2 != 0.f ? f2 * __builtin_fmaf(d2, l2, s2) : 0.f;
    l = l * f1 + l2 * f2; s = sa + sb; m = to;
  };
  float m = SM_NO_REF, l = 0.f, s = 0.f;
  for (int p = tid; p < a.parts; p += NT) { const float4 v = a.stats[(size_t)p * a.n + q]; join(m, l, s, v.x, v.y, v.z); }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) join(m, l, s, __shfl_xor(m, o), __shfl_xor(l, o), __shfl_xor(s, o));
  if (lane == 0) { s_m[wave] = m; s_l[wave] = l; s_a[wave] = s; }
  for (int c = tid; c < 512; c += NT) qs[c] = c < a.dim ? (float)qr[c] : 0.f;
  __syncthreads();
  m = s_m[0]; l = s_l[0]; s = s_a[0];
  for (int w = 1; w < NT / 64; ++w) join(m, l, s, s_m[w], s_l[w], s_a[w]);
  const double lse = (double)m * a.unscale + (double)logf(l);

  // ---- the answer's log probability, the entropy
  if (wave == 0) {
    const int t = a.targets ? a.targets[q] : -1;
    const bool has = t >= 0 && t < a.rows;
    const T* wr = W + (int64_t)(has ? t : 0) * a.w_stride;
    double dot = 0.0;
    for (int c = lane; c < a.dim; c += 64) dot = __builtin_fma((double)qs[c], (double)(float)wr[c], dot);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) dot += __shfl_xor(dot, o);
    if (lane == 0) {
      if (a.log_probs) a.log_probs[q] = !has ? 0.f : (is_allowed(t) ? (float)(dot * (double)a.scale - lse) : -__builtin_inff());
      if (a.entropy) a.entropy[q] = l == 0.f ? 0.f : fmaxf(logf(l) - MAR_LN2 * (s / l), 0.f);
    }
  }
  if (a.num_top == 0) return;

  // ---- groups with the largest maxima; among equal ones the first
  const int want = a.num_top + SM_MARGIN;
  const float* gm = a.gmax + q * a.ngroups;
  int have = 0;
  for (int64_t g0 = 0; g0 < a.ngroups; g0 += CHUNK) {
    const int n = (int)min((int64_t)CHUNK, a.ngroups - g0);
    for (int e = tid; e < n; e += NT) {
      const uint32_t k = order_key(gm[g0 + e]);
      keys[e] = k ? (unsigned long long)k << 32 | (uint32_t)~(uint32_t)(g0 + e) : 0ull;
    }
    for (int e = tid; e < have; e += NT) keys[n + e] = best[e];
    have = select_top<NT, CAP>(keys, n + have, want, cand, best, cnt);
  }
  for (int e = tid; e < have; e += NT) groups[e] = (int)~(uint32_t)best[e];
  __syncthreads();
  const int ngr = have, per = 16 * a.group_tiles;
  // ---- their rows in fp32, eight lanes to a row
  have = 0;
  const int64_t nrows = (int64_t)ngr * per;
  for (int64_t r0 = 0; r0 < nrows; r0 += CHUNK) {
    const int n = (int)min((int64_t)CHUNK, nrows - r0);
    for (int e = tid >> 3; e < (n + NT / 8 - 1) / (NT / 8) * (NT / 8); e += NT / 8) {
      bool in = e < n;
      int64_t row = 0;
      if (in) {
        const int64_t r = r0 + e;
        const int j = (int)(r / per), w = (int)(r - (int64_t)j * per), grp = groups[j], k = w & 15;
        row = ((int64_t)(grp >> 1) * a.group_tiles + (w >> 4)) * SM_TY + 8 * (k >> 2) + 4 * (grp & 1) + (k & 3);
        in = row < a.rows && is_allowed(row);
      }
      float sum = 0.f;
      if (in) {
        const T* wr = W + row * a.w_stride;
        for (int u = tid & 7; 8 * u < a.dim; u += 8) {
          float v[8];
          load8<TYPE>(wr, 8 * u, a.dim, v);
#pragma unroll
          for (int c = 0; c < 8; ++c) sum = __builtin_fmaf(v[c], qs[8 * u + c], sum);
        }
      }
      sum += __shfl_xor(sum, 1); sum += __shfl_xor(sum, 2); sum += __shfl_xor(sum, 4);
      if ((tid & 7) == 0 && e < n) {
        const uint32_t k = in ? order_key(sum) : 0u;
        keys[e] = k ? (unsigned long long)k << 32 | (uint32_t)~(uint32_t)row : 0ull;
      }
    }
    for (int e = tid; e < have; e += NT) keys[n + e] = best[e];
    have = select_top<NT, CAP>(keys, n + have, want, cand, best, cnt);
  }
  // ---- the best of them in 64 bits
  for (int e = wave; e < have; e += NT / 64) {
    const T* wr = W + (int64_t)(uint32_t)~(uint32_t)best[e] * a.w_stride;
    double dot = 0.0;
    for (int c = lane; c < a.dim; c += 64) dot = __builtin_fma((double)qs[c], (double)(float)wr[c], dot);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) dot += __shfl_xor(dot, o);
    if (lane == 0) exact[e] = dot;
  }
  __syncthreads();
  for (int e = tid; e < have; e += NT) {
    const double v = exact[e];
    const uint32_t row = ~(uint32_t)best[e];
    int rank = 0;
    for (int j = 0; j < have; ++j) rank += exact[j] > v || (exact[j] == v && ~(uint32_t)best[j] < row) ? 1 : 0;
    if (rank < a.num_top) {
      a.top_ids[q * a.num_top + rank] = (int32_t)row;
      a.top_log_probs[q * a.num_top + rank] = (float)(v * (double)a.scale - lse);
    }
  }
  for (int e = have + tid; e < a.num_top; e += NT) { a.top_ids[q * a.num_top + e] = -1; a.top_log_probs[q * a.num_top + e] = -__builtin_inff(); }
}

// ------------------------------------------------------------------------------------------ plan and checks -----
const char* sm_check(const mar_softmax* p, int* code) {
  *code = MAR_EINVAL;
  if (!p) return "problem is NULL";
  if (p->dtype < MAR_DTYPE_FP32 || p->dtype > MAR_DTYPE_FP16) return "unknown dtype";
  if (!(p->scale >= 1e-6f && p->scale <= 1e6f)) return "scale must lie in [1e-6, 1e6]";
  *code = MAR_ERANGE;
  if (p->num_rows < 1 || p->num_rows > MAR_SOFTMAX_MAX_ROWS) return "num_rows outside 1..MAR_SOFTMAX_MAX_ROWS";
  if (p->num_queries < 0 || p->num_queries > MAR_SOFTMAX_MAX_QUERIES) return "num_queries outside 0..MAR_SOFTMAX_MAX_QUERIES";
  if (p->dim < 1 || p->dim > MAR_MAX_DIM) return "dim outside 1..MAR_MAX_DIM";
  *code = MAR_EINVAL;
  if (p->row_stride < p->dim || p->query_stride < p->dim) return "a stride is below dim";
  if (p->row_stride > (int64_t)1 << 30 || p->query_stride > (int64_t)1 << 30) return "a stride is above 2^30";
  return nullptr;
}

// Parts: where the stripes do not fill the device, several workgroups share one, each streaming a part of the tiles.  Estimated by
// the rounds of workgroups and their tiles, a workgroup costing four tiles more for its rows and its first tile.
SmPlan sm_plan(int dtype, int dim, int pass, int64_t n_x, int64_t n_y, int multiple) {
  SmPlan r;
  const int nk = sm_nk(dim);
  r.qb = sm_qb(dtype, nk, pass);
  r.stripes = (int32_t)((n_x + 128 * r.qb - 1) / (128 * r.qb));
  r.ntiles = (int32_t)((n_y + SM_TY - 1) / SM_TY);
  const int64_t slots = 256 * sm_waves(dtype, nk, pass);
  int64_t best = INT64_MAX;
  r.parts = 1; r.tps = r.ntiles;
  const int most = pass == 0 ? 1024 : MAR_SOFTMAX_MAX_PARTS;
  for (int k = 1; k <= most && k <= r.ntiles; ++k) {
    int64_t tps = (r.ntiles + k - 1) / k;
    tps = (tps + multiple - 1) / multiple * multiple;
    const int64_t parts = (r.ntiles + tps - 1) / tps;
    const int64_t cost = (r.stripes * parts + slots - 1) / slots * (tps + (pass == 0 ? 4 : 8));
    if (cost < best) { best = cost; r.parts = (int32_t)parts; r.tps = (int32_t)tps; }
  }
  return r;
}

// Tiles to a group: about as many group maxima to look through as rows of the best groups to score again, in bytes.
static int group_tiles(const mar_softmax* p, int num_top) {
  const double ntiles = (double)((p->num_rows + SM_TY - 1) / SM_TY), row_bytes = p->dim * (p->dtype == MAR_DTYPE_FP32 ? 4.0 : 2.0);
  const double g = ntiles * 8.0 / ((num_top + SM_MARGIN) * 16.0 * row_bytes);
  int k = 1;
  while ((double)k * k < g) ++k;
  return k;
}

struct ProbsLayout { size_t stats, gmax, qtiles, qexps, wtiles, wexps, bytes; SmPlan p0; int group_tiles; int64_t ngroups; bool images; };
static ProbsLayout probs_layout(const mar_softmax* p, int num_top) {
  ProbsLayout L;
  L.group_tiles = num_top ? group_tiles(p, num_top) : 1;
  L.p0 = sm_plan(p->dtype, p->dim, 0, p->num_queries, p->num_rows, L.group_tiles);
  L.ngroups = num_top ? 2 * (int64_t)((L.p0.ntiles + L.group_tiles - 1) / L.group_tiles) : 0;
  const size_t T = (size_t)p->num_queries;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  L.stats = take((size_t)L.p0.parts * T * sizeof(float4));
  L.gmax = take(T * (size_t)L.ngroups * 4);
  L.images = L.p0.stripes >= MAR_SOFTMAX_IMAGES;
  L.qtiles = L.qexps = L.wtiles = L.wexps = at;
  if (L.images) {
    L.qtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_queries)); L.qexps = take(sm_exps_bytes(p->num_queries));
    L.wtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_rows)); L.wexps = take(sm_exps_bytes(p->num_rows));
  }
  L.bytes = at > 256 ? at : 256;
  return L;
}

template <int TYPE, bool IMG> static void launch_nk(const SmArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.units + 7) / 8 * 8)), block(256);
  switch (sm_nk(a.dim)) {
    case 2: hipLaunchKernelGGL((k_softmax<TYPE, 2, 0, IMG>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_softmax<TYPE, 4, 0, IMG>), grid, block, 0, st, a); break;
    case 7: hipLaunchKernelGGL((k_softmax<TYPE, 7, 0, IMG>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((k_softmax<TYPE, 8, 0, IMG>), grid, block, 0, st, a); break;
    case 12: hipLaunchKernelGGL((k_softmax<TYPE, 12, 0, IMG>), grid, block, 0, st, a); break;
    case 16: hipLaunchKernelGGL((k_softmax<TYPE, 16, 0, IMG>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_softmax<TYPE, 25, 0, IMG>), grid, block, 0, st, a); break;
  }
}
template <int TYPE> static void launch_pack(const SmPackArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.n + SM_TY - 1) / SM_TY)), block(256);
  switch (sm_nk(a.dim)) {
    case 2: hipLaunchKernelGGL((k_softmax_pack<TYPE, 2>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_softmax_pack<TYPE, 4>), grid, block, 0, st, a); break;
    case 7: hipLaunchKernelGGL((k_softmax_pack<TYPE, 7>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((k_softmax_pack<TYPE, 8>), grid, block, 0, st, a); break;
    case 12: hipLaunchKernelGGL((k_softmax_pack<TYPE, 12>), grid, block, 0, st, a); break;
    case 16: hipLaunchKernelGGL((k_softmax_pack<TYPE, 16>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_softmax_pack<TYPE, 25>), grid, block, 0, st, a); break;
  }
}
hipError_t sm_pack(int dtype, const SmPackArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_pack<0>(a, st); else if (dtype == MAR_DTYPE_BF16) launch_pack<1>(a, st); else launch_pack<2>(a, st);
  return hipGetLastError();
}
size_t sm_image_bytes(int dtype, int dim, int64_t rows) {
  const int nk = sm_nk(dim);
  return (size_t)((rows + SM_TY - 1) / SM_TY) * SM_TY * sp_pitch(nk) * (dtype == MAR_DTYPE_FP32 ? 2 : 1);
}
size_t sm_exps_bytes(int64_t rows) { return ((size_t)((rows + SM_TY - 1) / SM_TY) * 16 + 255) / 256 * 256; }
template <bool IMG> static hipError_t launch_stats(int dtype, const SmArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_nk<0, IMG>(a, st); else if (dtype == MAR_DTYPE_BF16) launch_nk<1, IMG>(a, st); else launch_nk<2, IMG>(a, st);
  return hipGetLastError();
}

// Few queries: a wide workgroup each; many: enough of them to fill the device at 256 threads.
template <int TYPE> static void launch_answer(const AnswerArgs& a, hipStream_t st) {
  if (a.n >= 512) hipLaunchKernelGGL((k_answer<TYPE, 256, 2048>), dim3((unsigned)a.n), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_answer<TYPE, 1024, 8192>), dim3((unsigned)a.n), dim3(1024), 0, st, a);
}

static bool top_ok(int32_t num_top) {
  if (num_top >= 0 && num_top <= MAR_MAX_TOP) return true;
  mar_set_error("num_top outside 0..%d", MAR_MAX_TOP);
  return false;
}

extern "C" int mar_log_probs_workspace_bytes(const mar_softmax* p, int32_t num_top, size_t* out_bytes) {
  int code;
  if (const char* why = sm_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (!top_ok(num_top)) return MAR_ERANGE;
  if (!out_bytes) { mar_set_error("out_bytes is NULL"); return MAR_EINVAL; }
  *out_bytes = probs_layout(p, num_top).bytes;
  return MAR_OK;
}

extern "C" int mar_log_probs(const mar_softmax* p, const void* queries, const void* table, const int32_t* targets, const uint32_t* allowed,
                             int64_t allowed_stride, int32_t num_top, float* log_probs, float* entropy, int32_t* top_ids,
                             float* top_log_probs, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int code;
  if (const char* why = sm_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (!top_ok(num_top)) return MAR_ERANGE;
  if (!table || (p->num_queries > 0 && !queries)) { mar_set_error("queries or table is NULL"); return MAR_EINVAL; }
  if (log_probs && !targets && p->num_queries > 0) { mar_set_error("log_probs needs targets"); return MAR_EINVAL; }
  if (num_top > 0 && p->num_queries > 0 && (!top_ids || !top_log_probs)) { mar_set_error("num_top needs top_ids and top_log_probs"); return MAR_EINVAL; }
  const uintptr_t align = p->dtype == MAR_DTYPE_FP32 ? 3 : 1;
  if (((uintptr_t)queries | (uintptr_t)table) & align) { mar_set_error("a matrix is not aligned to its type"); return MAR_EINVAL; }
  if (((uintptr_t)targets | (uintptr_t)allowed | (uintptr_t)log_probs | (uintptr_t)entropy | (uintptr_t)top_ids | (uintptr_t)top_log_probs) & 3) {
    mar_set_error("an array is not 4-byte aligned"); return MAR_EINVAL;
  }
  if (allowed && allowed_stride != 0 && allowed_stride < (p->num_rows + 31) / 32) { mar_set_error("allowed_stride is neither 0 nor a row of words"); return MAR_EINVAL; }
  if (!workspace || ((uintptr_t)workspace & 255)) { mar_set_error("workspace must be non-NULL and 256-byte aligned"); return MAR_EINVAL; }
  const ProbsLayout L = probs_layout(p, num_top);
  if (workspace_bytes < L.bytes) { mar_set_error("workspace has %zu bytes, %zu needed", workspace_bytes, L.bytes); return MAR_ENOMEM; }
  if (p->num_queries == 0) return MAR_OK;
  const hipStream_t st = (hipStream_t)hip_stream;
  SmArgs a = {};
  a.X = queries; a.x_stride = p->query_stride; a.n_x = p->num_queries;
  a.Y = table; a.y_stride = p->row_stride; a.n_y = (int32_t)p->num_rows;
  a.dim = p->dim; a.c = p->scale * 1.44269504088896341f;
  a.nstripes = L.p0.stripes; a.parts = L.p0.parts; a.tps = L.p0.tps; a.units = a.nstripes * a.parts;
  a.stats = (float4*)((char*)workspace + L.stats);
  a.gmax = num_top ? (float*)((char*)workspace + L.gmax) : nullptr;
  a.ngroups = L.ngroups; a.group_tiles = L.group_tiles;
  a.allowed = allowed; a.allowed_stride = allowed_stride;
  hipError_t e;
  if (L.images) {
    SmPackArgs k = {};
    k.dim = p->dim;
    k.src = table; k.stride = p->row_stride; k.n = (int32_t)p->num_rows; k.tiles = (char*)workspace + L.wtiles; k.exps = (int*)((char*)workspace + L.wexps);
    e = sm_pack(p->dtype, k, st);
    k.src = queries; k.stride = p->query_stride; k.n = p->num_queries; k.tiles = (char*)workspace + L.qtiles; k.exps = (int*)((char*)workspace + L.qexps);
    if (e == hipSuccess) e = sm_pack(p->dtype, k, st);
    if (e != hipSuccess) { mar_set_error("image kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
    a.ximg = {(char*)workspace + L.qtiles, (const int*)((char*)workspace + L.qexps)};
    a.yimg = {(char*)workspace + L.wtiles, (const int*)((char*)workspace + L.wexps)};
    e = launch_stats<true>(p->dtype, a, st);
  } else {
    e = launch_stats<false>(p->dtype, a, st);
  }
  if (e != hipSuccess) { mar_set_error("softmax kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  AnswerArgs r = {};
  r.Q = queries; r.W = table; r.q_stride = p->query_stride; r.w_stride = p->row_stride; r.rows = p->num_rows;
  r.n = p->num_queries; r.dim = p->dim; r.parts = L.p0.parts; r.num_top = num_top; r.group_tiles = L.group_tiles; r.ngroups = L.ngroups;
  r.scale = p->scale; r.unscale = (double)p->scale / (double)a.c;
  r.targets = targets; r.allowed = allowed; r.allowed_stride = allowed_stride; r.stats = a.stats; r.gmax = a.gmax;
  r.log_probs = log_probs; r.entropy = entropy; r.top_ids = top_ids; r.top_log_probs = top_log_probs;
  if (p->dtype == MAR_DTYPE_FP32) launch_answer<0>(r, st); else if (p->dtype == MAR_DTYPE_BF16) launch_answer<1>(r, st); else launch_answer<2>(r, st);
  e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("answer kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
