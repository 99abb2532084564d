// Rows drawn from scores with temperature, top-k, top-p and min-p (gfx950).
//
// Ranks are by (score descending, id ascending), so that every filter is a threshold: a key tau above which all rows are kept and a number
// of rows at tau, the first by id.  Weights are integers W = round(2^bits exp((s - max) / temperature)), bits such that their sum lies below
// 2^61: sums are exact in any order, and a border (top-p's, a draw's) falls where the integers say, for every kernel here alike.
#include "mar_sample_dev.h"

#define DRAW_SEGMENT 512                                    // columns of a segment: a wave's eight a lane

// Sums and maxima over a workgroup of 16 waves; everyone gets the result.
template <typename T, typename F> __device__ __forceinline__ T draw_reduce(T v, T* slots, F join) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = join(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  v = slots[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v = join(v, slots[w]);
  return v;
}
// Exclusive prefix sums over a workgroup; the whole sum in `total`.
template <typename T> __device__ __forceinline__ T draw_prefix(T v, T* slots, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T run = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const T up = __shfl_up(run, o); if (lane >= o) run += up; }
  __syncthreads();
  if (lane == 63) slots[wave] = run;
  __syncthreads();
  T before = 0, all = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) { if (w < wave) before += slots[w]; all += slots[w]; }
  total = all;
  return before + run - v;
}

// One workgroup a query.
template <int TYPE>
__global__ void __launch_bounds__(1024)
k_sample(DrawArgs a, int64_t first) {
  typedef typename RowType<TYPE>::T T;
  __shared__ draw_u64 bins[2048], slots[16];
  __shared__ unsigned found[2];
  __shared__ draw_u64 found_sum;
  const int64_t q = first + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = blockDim.x;
  const T* scores = (const T*)a.scores + q * a.score_stride;
  const uint32_t* allowed = a.allowed ? a.allowed + q * a.allowed_stride : nullptr;
  const DrawParams par = draw_params(a, q);
  auto max_of = [](unsigned x, unsigned y) { return x > y ? x : y; };
  auto sum_of = [](auto x, auto y) { return x + y; };

  // keys of columns c .. c + 7
  auto load = [&](int c, unsigned (&key)[8]) {
    float v[8];
    load8<TYPE>(scores, c, a.rows, v);
    const unsigned bits = allowed ? allowed[c >> 5] >> (c & 31) : 0xffu;
#pragma unroll
    for (int e = 0; e < 8; ++e) key[e] = c + e < a.rows && (bits >> e & 1u) ? draw_key(v[e]) : 0u;
  };
  auto each = [&](auto f) {
    for (int64_t c = 8 * tid; c < a.rows; c += 8 * threads) {
      unsigned key[8];
      load((int)c, key);
#pragma unroll
      for (int e = 0; e < 8; ++e) f(key[e]);
    }
  };

  unsigned best = 0, count = 0;
  each([&](unsigned k) { best = max(best, k); count += k != 0; });
  best = draw_reduce(best, (unsigned*)slots, max_of);
  count = draw_reduce(count, (unsigned*)slots, sum_of);
  if (count == 0) {                                        // uniform
    for (int d = tid; d < a.draws; d += threads) {
      a.ids[q * a.draws + d] = -1;
      if (a.log_probs) a.log_probs[q * a.draws + d] = -__builtin_inff();
    }
    if (tid == 0 && a.num_kept) a.num_kept[q] = 0;
    return;
  }
  const double top = (double)draw_score(best);
  auto distance = [&](unsigned k) { return ((double)draw_score(k) - top) * par.inv_temperature; };
  float approx = 0.f;
  each([&](unsigned k) { if (k) approx += __builtin_amdgcn_exp2f((float)(distance(k) * 1.4426950408889634)); });
  approx = draw_reduce(approx, (float*)slots, sum_of);
  const int bits = 60 - ilogbf(fmaxf(approx, 1.f));
  auto weight = [&](unsigned k) { return draw_weight(distance(k), bits); };

  // rows with a key above tau, and the first `at_tau` rows that have it
  unsigned tau = 0, at_tau = 0;
  // The largest key at which `of` summed over the keys from it upwards reaches `want`, by digits of 11, 11 and 10 bits; `above`: the
  // sum over greater keys.
  auto select = [&](draw_u64 want, unsigned least, auto of, draw_u64& above) {
    unsigned prefix = 0;
    draw_u64 over = 0;
    for (int level = 0; level < 3; ++level) {
      const int shift = level == 0 ? 21 : (level == 1 ? 10 : 0), width = level == 2 ? 10 : 11;
      for (int i = tid; i < 2048; i += threads) bins[i] = 0;
      __syncthreads();
      each([&](unsigned k) {
        if (k != 0 && k >= least && (level == 0 || k >> (shift + width) == prefix)) {
          const draw_u64 w = of(k);
          if (w) atomicAdd(&bins[k >> shift & ((1u << width) - 1)], w);
        }
      });
      __syncthreads();
      // thread i takes the i-th pair of bins from the top
      for (int i0 = 0; i0 < 1024; i0 += threads) {
        const int i = i0 + tid, hi = 2047 - 2 * i;
        const draw_u64 x = bins[hi], y = bins[hi - 1];
        draw_u64 all;
        const draw_u64 before = over + draw_prefix(x + y, slots, all);
        if (before < want && before + x + y >= want) {
          const bool one = before + x >= want;
          found[0] = (unsigned)(one ? hi : hi - 1);
          found_sum = before + (one ? 0 : x);
        }
        over += all;
      }
      __syncthreads();
      over = found_sum;
      prefix = prefix << width | found[0];
      __syncthreads();
    }
    above = over;
    return prefix;
  };
  if (par.top_k > 0 && (unsigned)par.top_k < count) {
    draw_u64 above;
    tau = select((draw_u64)par.top_k, 0, [](unsigned) { return (draw_u64)1; }, above);
    at_tau = (unsigned)(par.top_k - (int)above);
  }
  if (par.top_p < 2.f) {
    draw_u64 all = 0;
    each([&](unsigned k) { if (k > tau) all += weight(k); });
    all = draw_reduce(all, slots, sum_of) + (tau ? at_tau * weight(tau) : 0);
    draw_u64 want = draw_share_up(par.top_p, all);
    if (want == 0) want = 1;
    // rows at the border of top-k count fully here: the sum is reached at that key at the latest, and its rows are counted below
    draw_u64 above;
    const unsigned border = select(want, tau, [&](unsigned k) { return weight(k); }, above);
    const draw_u64 w = weight(border);
    tau = border; at_tau = (unsigned)((want - above + w - 1) / w);
  }
  const draw_u64 least = par.min_p > 0.f ? (draw_u64)__builtin_ceil(__builtin_ldexp((double)par.min_p, bits)) : 0;
  const draw_u64 w_tau = tau ? weight(tau) : 0;

  // mass above tau and rows at tau, segment by segment
  draw_u64* mass = a.mass + q * a.segments;
  uint32_t* ties = a.ties + q * a.segments;
  unsigned kept = 0;
  for (int seg = wave; seg < a.segments; seg += threads >> 6) {
    const int64_t c = (int64_t)seg * DRAW_SEGMENT + 8 * lane;
    draw_u64 sum = 0;
    unsigned same = 0;
    if (c < a.rows) {
      unsigned key[8];
      load((int)c, key);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (key[e] > tau) { const draw_u64 w = weight(key[e]); if (w >= least) { sum += w; ++kept; } }
        same += tau != 0 && key[e] == tau;
      }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) { sum += __shfl_xor(sum, o); same += __shfl_xor(same, o); }
    if (lane == 0) { mass[seg] = sum; ties[seg] = same; }
  }
  kept = draw_reduce(kept, (unsigned*)slots, sum_of);
  if (tid == 0 && a.num_kept) a.num_kept[q] = (int)(kept + (tau && w_tau >= least ? at_tau : 0));
  if (w_tau < least) at_tau = 0;
  __syncthreads();
  // prefixes: rows at tau before the segment, mass before it
  draw_u64 total = 0;
  unsigned before_ties = 0;
  for (int s0 = 0; s0 < a.segments; s0 += threads) {
    const int seg = s0 + tid;
    const unsigned mine = seg < a.segments ? ties[seg] : 0;
    unsigned all_ties;
    const unsigned before = before_ties + draw_prefix(mine, (unsigned*)slots, all_ties);
    before_ties += all_ties;
    const unsigned taken = before >= at_tau ? 0 : min(mine, at_tau - before);
    draw_u64 all;
    const draw_u64 m = (seg < a.segments ? mass[seg] : 0) + taken * w_tau;
    const draw_u64 start = total + draw_prefix(m, slots, all);
    total += all;
    if (seg < a.segments) { mass[seg] = start; ties[seg] = before; }
  }
  __syncthreads();
  // a wave a draw
  const double log_total = log(__builtin_ldexp((double)total, -bits));
  for (int d = wave; d < a.draws; d += threads >> 6) {
    const float u = a.uniforms[q * a.draws + d];
    draw_u64 target = !(u > 0.f) ? 0 : (u >= 1.f ? total - 1 : draw_share_down(u, total));
    int lo = 0, hi = a.segments;                           // the last segment that begins at or below the target
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (mass[mid] <= target) lo = mid; else hi = mid; }
    target -= mass[lo];
    const int64_t c = (int64_t)lo * DRAW_SEGMENT + 8 * lane;
    unsigned key[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    if (c < a.rows) load((int)c, key);
    unsigned same = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) same += tau != 0 && key[e] == tau;
    unsigned rank = same;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const unsigned up = __shfl_up(rank, o); if (lane >= o) rank += up; }
    rank += ties[lo] - same;
    draw_u64 w[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = 0;
      if (key[e] > tau) { w[e] = weight(key[e]); if (w[e] < least) w[e] = 0; }
      else if (tau != 0 && key[e] == tau) { if (rank < at_tau) w[e] = w_tau; ++rank; }
      sum += w[e];
    }
    draw_u64 run = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const draw_u64 up = __shfl_up(run, o); if (lane >= o) run += up; }
    draw_u64 start = run - sum;
    if (start <= target && target < run) {                 // one lane
      int e = 0;
      unsigned k = key[0];
      draw_u64 at = start + w[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) if (at <= target) { at += w[j]; e = j; k = key[j]; }
      a.ids[q * a.draws + d] = (int)c + e;
      if (a.log_probs) a.log_probs[q * a.draws + d] = (float)(distance(k) - log_total);
    }
  }
}

// ------------------------------------------------------------------------------------------ entry points -----
static const char* draw_check(const mar_sampling* p, int* code) {
  *code = MAR_EINVAL;
  if (!p) return "problem is NULL";
  if (p->reserved != 0) return "reserved must be 0";
  if (p->dtype < MAR_DTYPE_FP32 || p->dtype > MAR_DTYPE_FP16) return "unknown dtype";
  if (!(p->temperature >= 0.f)) return "temperature must be 0 or above";
  if (p->top_k < 0) return "top_k must be 0 or above";
  if (!(p->top_p >= 0.f && p->top_p <= 1.f)) return "top_p must lie in 0 .. 1";
  if (!(p->min_p >= 0.f && p->min_p <= 1.f)) return "min_p must lie in 0 .. 1";
  *code = MAR_ERANGE;
  if (p->num_rows < 1 || p->num_rows > MAR_SOFTMAX_MAX_ROWS) return "num_rows outside 1..MAR_SOFTMAX_MAX_ROWS";
  if (p->num_queries < 0 || p->num_queries > MAR_SOFTMAX_MAX_QUERIES) return "num_queries outside 0..MAR_SOFTMAX_MAX_QUERIES";
  if (p->num_draws < 1 || p->num_draws > MAR_MAX_DRAWS) return "num_draws outside 1..MAR_MAX_DRAWS";
  *code = MAR_EINVAL;
  if (p->score_stride < p->num_rows || p->score_stride > (int64_t)1 << 40) return "score_stride is below num_rows or above 2^40";
  return nullptr;
}
struct DrawLayout { size_t mass, ties, bytes; int segments; };
static DrawLayout draw_layout(const mar_sampling* p) {
  DrawLayout L;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  L.segments = (int)((p->num_rows + DRAW_SEGMENT - 1) / DRAW_SEGMENT);
  L.mass = take((size_t)p->num_queries * L.segments * 8);
  L.ties = take((size_t)p->num_queries * L.segments * 4);
  L.bytes = at > 256 ? at : 256;
  return L;
}

extern "C" int mar_sample_rows_workspace_bytes(const mar_sampling* p, size_t* out_bytes) {
  int code;
  if (const char* why = draw_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (!out_bytes) { mar_set_error("out_bytes is NULL"); return MAR_EINVAL; }
  *out_bytes = draw_layout(p).bytes;
  return MAR_OK;
}

extern "C" int mar_sample_rows(const mar_sampling* p, const void* scores, const uint32_t* allowed, int64_t allowed_stride,
                               const float* temperatures, const int32_t* top_ks, const float* top_ps, const float* min_ps, const float* uniforms,
                               int32_t* ids, float* log_probs, int32_t* num_kept, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int code;
  if (const char* why = draw_check(p, &code)) { mar_set_error("%s", why); return code; }
  if (p->num_queries > 0 && (!scores || !uniforms || !ids)) { mar_set_error("scores, uniforms or ids is NULL"); return MAR_EINVAL; }
  if ((uintptr_t)scores & (p->dtype == MAR_DTYPE_FP32 ? 3 : 1)) { mar_set_error("scores is not aligned to its type"); return MAR_EINVAL; }
  if (((uintptr_t)allowed | (uintptr_t)temperatures | (uintptr_t)top_ks | (uintptr_t)top_ps | (uintptr_t)min_ps | (uintptr_t)uniforms | (uintptr_t)ids |
       (uintptr_t)log_probs | (uintptr_t)num_kept) & 3) { mar_set_error("an array is not 4-byte aligned"); return MAR_EINVAL; }
  if (allowed && allowed_stride != 0 && allowed_stride < (p->num_rows + 31) / 32) { mar_set_error("allowed_stride is neither 0 nor a row of words"); return MAR_EINVAL; }
  if (!workspace || ((uintptr_t)workspace & 255)) { mar_set_error("workspace must be non-NULL and 256-byte aligned"); return MAR_EINVAL; }
  const DrawLayout L = draw_layout(p);
  if (workspace_bytes < L.bytes) { mar_set_error("workspace has %zu bytes, %zu needed", workspace_bytes, L.bytes); return MAR_ENOMEM; }
  if (p->num_queries == 0) return MAR_OK;
  DrawArgs a = {};
  a.scores = scores; a.allowed = allowed; a.temperatures = temperatures; a.top_ks = top_ks; a.top_ps = top_ps; a.min_ps = min_ps; a.uniforms = uniforms;
  a.ids = ids; a.log_probs = log_probs; a.num_kept = num_kept; a.score_stride = p->score_stride; a.allowed_stride = allowed_stride;
  a.rows = (int32_t)p->num_rows; a.draws = p->num_draws; a.segments = L.segments;
  a.top_k = p->top_k; a.temperature = p->temperature; a.top_p = p->top_p; a.min_p = p->min_p;
  a.mass = (draw_u64*)((char*)workspace + L.mass); a.ties = (uint32_t*)((char*)workspace + L.ties);
  const hipStream_t st = (hipStream_t)hip_stream;
  sm_launches(p->num_queries, 1024, [&](int64_t first, unsigned blocks) {
    if (p->dtype == MAR_DTYPE_FP32) hipLaunchKernelGGL(k_sample<0>, dim3(blocks), dim3(1024), 0, st, a, first);
    else if (p->dtype == MAR_DTYPE_BF16) hipLaunchKernelGGL(k_sample<1>, dim3(blocks), dim3(1024), 0, st, a, first);
    else hipLaunchKernelGGL(k_sample<2>, dim3(blocks), dim3(1024), 0, st, a, first);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("sampling kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
