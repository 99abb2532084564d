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

// A row's place in the order (score descending, id ascending) as one number: greater comes first.  0: the row does not count.
__device__ __forceinline__ draw_u64 draw_place(unsigned key, unsigned id) { return (draw_u64)key << 32 | (key ? ~id : 0u); }

#define DRAW_SEGMENT 512            // columns of a segment: a wave's eight a lane
#define DRAW_SMALL (16 * 1024)      // rows that a workgroup holds in registers
#define DRAW_BINS 2048              // of weights: 1/32 of a binary order of magnitude each; the last one holds all below 2^-64 too
#define DRAW_FEW 1024               // largest top-k whose rows are picked from groups' maxima
#define DRAW_LIST 8192              // most rows a border is looked for among
#define DRAW_LIST_CHUNK 2048        // of one chunk

struct DrawChunk { unsigned best, count; float sum; };      // of a chunk: greatest key, rows that count, sum of weights relative to `best`
// Of a query, after the histogram: bins below `low` lie above top-p's border, bins above `high` below it.
struct DrawRange { int low, high; };

struct DrawArgs {
  const void* scores; const uint32_t* allowed;
  const float* temperatures; const int32_t* top_ks; const float *top_ps, *min_ps, *uniforms;
  int32_t* ids; float* log_probs; int32_t* num_kept;
  int64_t score_stride, allowed_stride;
  int32_t rows, draws, segments;
  int32_t top_k; float temperature, top_p, min_p;
  int32_t chunks, chunk_rows;       // of a query; a multiple of 2,048 rows
  int32_t blocks, groups;           // groups of rows a thread of the scan takes in a chunk, of a query in all
  int32_t list;                     // places in a query's list
  DrawChunk* stats;                 // [queries][chunks]
  unsigned* maxima;                 // [queries][groups]
  unsigned* hist;                   // [queries][chunks][DRAW_BINS], in units of 2^-hist_bits of the bin's largest weight
  int32_t hist_bits;
  DrawRange* range;                 // [queries]
  draw_u64* totals;                 // [queries][chunks][2]: sum of all weights, of those kept above the range
  unsigned* kept;                   // [queries][chunks]: rows kept above the range
  unsigned* listed;                 // [queries]: rows in the list (more than there are places: it does not serve)
  draw_u64* lists;                  // [queries][list]
  draw_u64* mass;                   // [queries][segments]
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
// Ways of a query: rows picked from groups' maxima, or all rows weighed, with a histogram where top-p's border is looked for.
__device__ __forceinline__ bool draw_few(const DrawArgs& a, const DrawParams& p) { return p.top_k > 0 && p.top_k <= DRAW_FEW && 2 * p.top_k <= a.groups; }
__device__ __forceinline__ bool draw_all(const DrawArgs& a, const DrawParams& p) { return p.top_k == 0 || p.top_k >= a.rows; }

// Keys of a query's columns, eight at a time.
template <int TYPE> struct DrawRow {
  typedef typename RowType<TYPE>::T T;
  const T* scores; const uint32_t* allowed; int rows;
  __device__ __forceinline__ DrawRow(const DrawArgs& a, int64_t q)
      : scores((const T*)a.scores + q * a.score_stride), allowed(a.allowed ? a.allowed + q * a.allowed_stride : nullptr), rows(a.rows) {}
  __device__ __forceinline__ void keys(int c, unsigned (&key)[8]) const {           // c < rows
    float v[8];
    load8<TYPE>(scores, c, rows, v);
    const unsigned bits = allowed ? allowed[c >> 5] >> (c & 31) : 0xffu;
#pragma unroll
    for (int e = 0; e < 8; ++e) key[e] = c + e < rows && (bits >> e & 1u) ? draw_key(v[e]) : 0u;
  }
};

// Weights of a query's rows: the best score, the inverse temperature, the integers' scale.
struct DrawWeights {
  double top, inv_temperature; int bits;
  __device__ __forceinline__ double distance(unsigned key) const { return ((double)draw_score(key) - top) * inv_temperature; }
  __device__ __forceinline__ draw_u64 of(unsigned key) const { return draw_weight(distance(key), bits); }
  // min-p's weight
  __device__ __forceinline__ draw_u64 least(float min_p) const { return min_p > 0.f ? (draw_u64)__builtin_ceil(__builtin_ldexp((double)min_p, bits)) : 0; }
};
// approx: sum of weights relative to the best one, in fp32: the integers' sum lies below 2^61 and a little more.
__device__ __forceinline__ DrawWeights draw_weights(unsigned best, const DrawParams& p, float approx) {
  return {(double)draw_score(best), p.inv_temperature, 60 - ilogbf(fmaxf(approx, 1.f))};
}
// The same in fp32 and binary orders of magnitude below the best, for sums that only choose a scale or a range of bins.
__device__ __forceinline__ float draw_depth(float top, float s, float c) { return fminf(top - s, 3.402823466e38f) * c; }
__device__ __forceinline__ float draw_depth_scale(const DrawParams& p) { return (float)fmin(p.inv_temperature * 1.4426950408889634, 3e38); }
__device__ __forceinline__ int draw_bin(float depth) { return (int)fminf(depth * 32.f, DRAW_BINS - 1.f); }
__device__ __forceinline__ draw_u64 draw_one() { return 1; }

// Sums and maxima over a workgroup; everyone gets the result.  slots: one a wave.
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
template <typename T> __device__ __forceinline__ T draw_sum(T v, T* slots) { return draw_reduce(v, slots, [](T x, T y) { return x + y; }); }
template <typename T> __device__ __forceinline__ T draw_wave_prefix(T v) {                // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const T up = __shfl_up(v, o); if (lane >= o) v += up; }
  return v;
}
// Exclusive prefix sums over a workgroup; the whole sum in `total`.
template <typename T> __device__ __forceinline__ T draw_prefix(T v, T* slots, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T run = draw_wave_prefix(v);
  __syncthreads();
  if (lane == 63) slots[wave] = run;
  __syncthreads();
  T before = 0, all = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) { if (w < wave) before += slots[w]; all += slots[w]; }
  total = all;
  return before + run - v;
}

// LDS of a workgroup of 1,024 threads that looks for a border.
struct DrawShared {
  draw_u64 bins[2048], slots[16], found_sum, found_all;
  unsigned found;
};
// The place of the first row, in the order of places, at which the sum of the rows' weights up to it reaches `want`; `over`: what lies
// above all rows that `each` goes through.  By digits of 11, 11 and 10 bits of the keys and, where several rows share the border's key, of
// the ids.  All 1,024 threads call it; each(f) calls f(place, weight) for every row of the thread, weight() its weight, of(key) that of a key.
template <typename E, typename W>
__device__ __forceinline__ draw_u64 draw_border(DrawShared& lds, draw_u64 want, draw_u64 over, E each, W of) {
  draw_u64 prefix = 0;
  for (int level = 0; level < 6; ++level) {
    const int width = level % 3 == 2 ? 10 : 11, shift = (level < 3 ? 32 : 0) + (level % 3 == 0 ? 21 : (level % 3 == 1 ? 10 : 0));
    for (int i = threadIdx.x; i < 2048; i += 1024) lds.bins[i] = 0;
    __syncthreads();
    each([&](draw_u64 place, auto weight) {
      if (place != 0 && (level == 0 || place >> (shift + width) == prefix)) {
        const draw_u64 w = weight();
        if (w) atomicAdd(&lds.bins[place >> shift & ((1u << width) - 1)], w);
      }
    });
    __syncthreads();
    const int hi = 2047 - 2 * (int)threadIdx.x;            // a pair of bins a thread, from the top
    const draw_u64 x = lds.bins[hi], y = lds.bins[hi - 1];
    draw_u64 all;
    const draw_u64 before = over + draw_prefix(x + y, lds.slots, all);
    if (before < want && before + x + y >= want) {
      const bool one = before + x >= want;
      lds.found = (unsigned)(one ? hi : hi - 1);
      lds.found_sum = before + (one ? 0 : x);
      lds.found_all = one ? x : y;
    }
    __syncthreads();
    over = lds.found_sum;
    prefix = prefix << width | lds.found;
    const draw_u64 ties = lds.found_all;
    __syncthreads();
    // all rows at the key are needed: no id decides
    if (level == 2 && want - over > ties - of((unsigned)prefix)) return prefix << 32;
  }
  return prefix;
}
