// Draws from scores (gfx950): ranking keys and integer weights, shared by the kernels of mar_sample.hip.
#pragma once
#include "mar_common.h"
#include "mar_rows_dev.h"
#include "mar_softmax.h"

typedef unsigned long long draw_u64;

// Scores as unsigned integers in their order; 0: the row does not count (-infinity).  -0 and 0 are one.
__device__ __forceinline__ unsigned draw_key(float s) {
  if (!(s > -__builtin_inff())) return 0u;
  const unsigned b = __float_as_uint(s + 0.f);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float draw_score(unsigned key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// round(2^(62 - shift - depth)), depth >= 0 (not a number, or 64 and more: 0), to 2^-51 of itself: 1 + 2^-(1/2 + g), |g| <= 1/2, by the
// polynomial of degree 10 through its Chebyshev series (off by 2^-52.5), whose bits less those of 1 are the power in units of 2^-52.
// The coefficients come from memory: out of scalar registers they are an operand of the products, constants would be copied for each.
static __constant__ double draw_power[11] = {1.7071067811865475, -0.4901290717342769, 0.1698657920915381, -0.039247331620345965, 0.006801044314302664,
                                             -0.0009428249441899351, 0.0001089194084511562, -1.0785257377670457e-05, 9.344721961284408e-07,
                                             -7.21863451712333e-08, 5.002210946656729e-09};
__device__ __forceinline__ draw_u64 draw_weight(double depth, int shift) {
  depth = fmin(depth, 64.0);
  const double g = __builtin_amdgcn_fract(depth) - 0.5;
  double p = draw_power[10];
#pragma unroll
  for (int i = 9; i >= 0; --i) p = __builtin_fma(p, g, draw_power[i]);
  const draw_u64 m = ((draw_u64)__double_as_longlong(p) - 0x3ff0000000000000ull) << 10;      // up to 2^62
  return ((m >> min((int)depth + (shift - 1), 63)) + 1) >> 1;          // shift >= 2
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

#define DRAW_TOP 3.402823466e38f    // the largest float
#define DRAW_SEGMENT 512            // columns of a segment: a wave's eight a lane
#define DRAW_SMALL (16 * 1024)      // rows that a workgroup holds in registers
#define DRAW_BINS 2048              // of weights: 1/32 of a binary order of magnitude each, or less (draw_fine)
#define DRAW_FEW 2048               // largest top-k whose rows are picked from groups' maxima
#define DRAW_LIST 8192              // rows of a border that a workgroup holds
#define DRAW_LIST_CHUNK 2048        // of one chunk

// Of a chunk: greatest key (0: no row counts), complement of the least one that weighs something beside it (0: not looked for), sum of weights
// relative to the best (where no histogram gives it).
struct DrawChunk { unsigned best, low; float sum; };
// Of a query, after the histogram: bins below `low` lie above top-p's border, bins above `high` below it; the sum of weights.
struct DrawRange { int low, high; float sum; };

struct DrawArgs {
  const void* scores; const uint32_t* allowed;
  const float* temperatures; const int32_t* top_ks; const float *top_ps, *min_ps, *uniforms;
  int32_t* ids; float* log_probs; int32_t* num_kept;
  int64_t score_stride, allowed_stride;
  int32_t rows, draws, segments;
  int32_t top_k; float temperature, top_p, min_p;
  int32_t chunks, chunk_rows;       // of a query; a multiple of 2,048 rows
  int32_t blocks, merge, groups;    // groups of rows a thread of the scan takes in a chunk, threads that share one, of a query in all
  int32_t list;                     // places in a query's list
  DrawChunk* stats;                 // [queries][chunks]
  unsigned* maxima;                 // [queries][groups]
  unsigned* hist;                   // [queries][chunks][DRAW_BINS], in units of 2^-hist_bits of the bin's largest weight
  int32_t hist_bits;
  DrawRange* range;                 // [queries]
  draw_u64* totals;                 // [queries][chunks][2]: sum of all weights, of those kept above the range
  unsigned* kept;                   // [queries][chunks]: rows kept above the range
  unsigned* listed;                 // [queries]: rows in the list (more than there are places: it does not serve)
  unsigned* undone;                 // [queries]: left to the last kernel
  draw_u64* lists;                  // [queries][list]
  draw_u64* mass;                   // [queries][mass_pitch]: sums of weights kept in segments
  int32_t mass_pitch;
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
// What a row may score below the best one for min-p to keep it; infinite: off, or an infinite temperature.  One wave finds it for all, before the first barrier: logarithm and
// division in every wave took 1,000 x 16,000 with min-p from 36.4 to 38.0 us.
__device__ __forceinline__ double draw_drop(const DrawParams& p) {
  if (!(p.min_p > 0.f)) return __builtin_inf();
  const double drop = -log((double)p.min_p) / p.inv_temperature;
  return drop >= 0.0 ? drop : __builtin_inf();
}
// Ways of a query: rows picked from groups' maxima, or all rows weighed, with a histogram where top-p's border is looked for.
// Picked: as many groups as top-k are enough for a bound; some G ln(1 / (1 - top_k / G)) rows reach it.
__host__ __device__ inline bool draw_picks(int top_k, int groups) { return top_k > 0 && top_k <= DRAW_FEW && top_k <= groups; }
__device__ __forceinline__ bool draw_few(const DrawArgs& a, const DrawParams& p) { return draw_picks(p.top_k, a.groups); }
__device__ __forceinline__ bool draw_all(const DrawArgs& a, const DrawParams& p) { return p.top_k == 0 || p.top_k >= a.rows; }
// Whose best score is infinite (or the largest float) goes by digits: the passes over all rows take their values as they are.
__device__ __forceinline__ bool draw_infinite(unsigned best) { return best >= 0xff7fffffu; }

// Keys of a query's columns, eight at a time.
template <int TYPE> struct DrawRow {
  typedef typename RowType<TYPE>::T T;
  const T* scores; const uint32_t* allowed; int rows;
  __device__ __forceinline__ DrawRow(const DrawArgs& a, int64_t q)
      : scores((const T*)a.scores + q * a.score_stride), allowed(a.allowed ? a.allowed + q * a.allowed_stride : nullptr), rows(a.rows) {}
  // c < rows.  -infinity: the row does not count, as where NaN is left
  __device__ __forceinline__ void raw(int c, float (&v)[8]) const {
    load8<TYPE>(scores, c, rows, v);
    unsigned bits = allowed ? allowed[c >> 5] >> (c & 31) : 0xffu;
    if (c + 8 > rows) bits &= 0xffu >> (c + 8 - rows);
    if ((bits & 0xffu) != 0xffu) {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (!(bits >> e & 1u)) v[e] = -__builtin_inff();
    }
  }
  // Without NaN, and +infinity as the largest float.
  __device__ __forceinline__ void scores_of(int c, float (&v)[8]) const {
    raw(c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fminf(fmaxf(v[e], -__builtin_inff()), DRAW_TOP);    // NaN gives way
  }
  __device__ __forceinline__ void keys(int c, unsigned (&key)[8]) const {
    float v[8];
    scores_of(c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) key[e] = draw_key(v[e]);
  }
};

// Weights of a query's rows: the best score, the inverse temperature and the same in binary orders of magnitude, the integers' scale 2^(62 - shift).
struct DrawWeights {
  double top, inv_temperature, slope; int shift;
  __device__ __forceinline__ draw_u64 of_score(float score) const { return draw_weight((top - (double)score) * slope, shift); }
  __device__ __forceinline__ draw_u64 of(unsigned key) const { return of_score(draw_score(key)); }
  __device__ __forceinline__ double log_sum(draw_u64 sum) const { return log(__builtin_ldexp((double)sum, shift - 62)); }
  // The best row's weight is a power of two less its rounding: a row that is certain keeps log 1.
  __device__ __forceinline__ float log_prob(unsigned key, double log_sum) const {
    return (float)fmin(((double)draw_score(key) - top) * inv_temperature - log_sum, 0.0);
  }
  // The least score that min-p keeps, rounded up: it tells rows apart whose integers are 0 too.
  __device__ __forceinline__ float floor(double drop) const {
    const double least = fmax(top - drop, -(double)DRAW_TOP);
    const float s = (float)least;
    return (double)s < least ? draw_score(draw_key(s) + 1) : s;
  }
};
// approx: sum of weights relative to the best one, in fp32: the integers' sum
// lies between 2^60 and 2^61, or a little more.
__device__ __forceinline__ DrawWeights draw_weights(unsigned best, const DrawParams& p, float approx) {
  return {(double)draw_score(best), p.inv_temperature, p.inv_temperature * 1.4426950408889634, 2 + ilogbf(fmaxf(approx, 1.f))};
}
// The same in fp32 and binary orders of magnitude below the best, for sums that only choose a scale or a range of bins.
__device__ __forceinline__ float draw_depth(float top, float s, float c) { return fminf(top - s, DRAW_TOP) * c; }
// What scores further below the best weigh less than 2^-63 of it.
__device__ __forceinline__ float draw_window(float c) { return 63.f / c; }
__device__ __forceinline__ float draw_depth_scale(const DrawParams& p) { return (float)fmin(p.inv_temperature * 1.4426950408889634, 3e38); }
// A weight relative to the best in units of 2^-18, and the sum of up to 8,192 of them: the same whatever order a list's rows have got.
__device__ __forceinline__ unsigned draw_part(float top, unsigned key, float c) { return (unsigned)(__builtin_amdgcn_exp2f(-draw_depth(top, draw_score(key), c)) * 0x1p18f); }
__device__ __forceinline__ float draw_parts(unsigned sum) { return (float)sum * 0x1p-18f; }
__device__ __forceinline__ draw_u64 draw_one() { return 1; }

// Sums and maxima by lane exchanges within a wave, zeros beyond its ends.
template <int CTRL, int ROWS, typename T> __device__ __forceinline__ T draw_moved(T v) {
  unsigned w[(sizeof(T) + 3) / 4];
  __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)w[i], CTRL, ROWS, 0xf, false);
  __builtin_memcpy(&v, w, sizeof(T));
  return v;
}
template <typename T> __device__ __forceinline__ T draw_lane(T v, int lane) {             // lane: uniform
  unsigned w[(sizeof(T) + 3) / 4];
  __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = (unsigned)__builtin_amdgcn_readlane((int)w[i], lane);
  __builtin_memcpy(&v, w, sizeof(T));
  return v;
}
struct DrawAdd { template <typename T> __device__ __forceinline__ T operator()(T x, T y) const { return x + y; } };
struct DrawMax { template <typename T> __device__ __forceinline__ T operator()(T x, T y) const { return x > y ? x : y; } };
template <typename J, typename T> __device__ __forceinline__ T draw_row_prefix(T v, J join) {         // inclusive, within 16 lanes
  v = join(v, draw_moved<0x111, 0xf>(v));
  v = join(v, draw_moved<0x112, 0xf>(v));
  v = join(v, draw_moved<0x114, 0xf>(v));
  return join(v, draw_moved<0x118, 0xf>(v));
}
template <typename J, typename T> __device__ __forceinline__ T draw_wave_prefix(T v, J join) {        // inclusive; zero is the joining's own
  v = draw_row_prefix(v, join);
  v = join(v, draw_moved<0x142, 0xa>(v));                  // lane 15 of rows 0 and 2 to rows 1 and 3
  return join(v, draw_moved<0x143, 0xc>(v));               // lane 31 to rows 2 and 3
}
template <typename T> __device__ __forceinline__ T draw_wave_prefix(T v) { return draw_wave_prefix(v, DrawAdd()); }
template <typename T> __device__ __forceinline__ T draw_wave_sum(T v) { return draw_lane(draw_wave_prefix(v, DrawAdd()), 63); }
// Over a workgroup of up to 16 waves; everyone gets the result.  slots: one a wave.
template <typename J, typename T> __device__ __forceinline__ T draw_reduce(T v, T* slots, J join) {
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  v = draw_wave_prefix(v, join);
  __syncthreads();
  if (lane == 63) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  T each = 0;
  if ((lane & 15) < waves) each = slots[lane & 15];
  return draw_lane(draw_row_prefix(each, join), 15);
}
template <typename T> __device__ __forceinline__ T draw_sum(T v, T* slots) { return draw_reduce(v, slots, DrawAdd()); }
// Exclusive prefix sums over a workgroup; the whole sum in `total`.
template <typename T> __device__ __forceinline__ T draw_prefix(T v, T* slots, T& total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const T run = draw_wave_prefix(v);
  __syncthreads();
  if (lane == 63) slots[wave] = run;
  __syncthreads();
  T each = 0;
  if ((lane & 15) < waves) each = slots[lane & 15];
  each = draw_row_prefix(each, DrawAdd());
  total = draw_lane(each, 15);
  const T before = wave ? draw_lane(each, wave - 1) : T(0);
  return before + run - v;
}

// LDS of up to 256 rows, each compared with all others by four of 1,024 threads.
#define DRAW_SHORT 256
struct DrawShort {
  struct { draw_u64 place, weight; } row[DRAW_SHORT];
  draw_u64 start[DRAW_SHORT], slots[16];
  unsigned id[DRAW_SHORT];
  float log_prob[DRAW_SHORT];
};
// The row of up to 256 at which the sum of weights reaches `want`, `over` above them.  place(i): of row i; of(key): a key's weight.
template <typename P, typename W>
__device__ __forceinline__ draw_u64 draw_border_short(DrawShort& lds, unsigned n, draw_u64 want, draw_u64 over, P place, W of) {
  const unsigned tid = threadIdx.x, r = tid >> 2, part = tid & 3, padded = (n + 15) & ~15u;
  if (tid < padded) {
    const draw_u64 p = tid < n ? place(tid) : 0;
    lds.row[tid] = {p, p ? of((unsigned)(p >> 32)) : 0};
  }
  __syncthreads();
  const draw_u64 mine = r < n ? lds.row[r].place : 0, weight = r < n ? lds.row[r].weight : 0;
  draw_u64 before = 0;
#pragma unroll 4
  for (unsigned i = part; i < padded; i += 4) {
    const auto other = lds.row[i];
    before += other.place > mine ? other.weight : 0;
  }
  before += draw_moved<0xB1, 0xf>(before);                 // over the four threads of a row: lanes 1 0 3 2, then 2 3 0 1
  before += draw_moved<0x4E, 0xf>(before) + over;
  if (part == 0 && before < want && before + weight >= want) lds.slots[0] = mine;      // one row
  __syncthreads();
  return lds.slots[0];
}

#define DRAW_DIGIT 12               // bits of a border's digit: 24 bits of range take two
// LDS of a workgroup of 1,024 threads that looks for a border.
struct DrawShared {
  draw_u64 bins[1 << DRAW_DIGIT], slots[16], found_sum, found_all;
  unsigned found, listed, ends[4][16];
};
static_assert(sizeof(DrawShort) + DRAW_SHORT * sizeof(draw_u64) <= sizeof(draw_u64) << DRAW_DIGIT, "the border's rows and their list in the digits' place");
// Adds a wave's weights to their bins.  Lanes that share a bin add up first, as long as many do: additions to one address go one by one.
__device__ __forceinline__ void draw_add(DrawShared& lds, bool has, unsigned bin, draw_u64 w) {
  draw_u64 left = __builtin_amdgcn_ballot_w64(has);
  for (int turn = 0; turn < 4 && left; ++turn) {           // uniform
    const unsigned one = (unsigned)__builtin_amdgcn_readlane((int)bin, __ffsll((long long)left) - 1);
    const bool same = has && bin == one;
    const draw_u64 lanes = __builtin_amdgcn_ballot_w64(same);
    if (__popcll(lanes) < 6) break;
    const draw_u64 sum = draw_wave_sum(same ? w : 0);
    if ((int)(threadIdx.x & 63) == __ffsll((long long)lanes) - 1) atomicAdd(&lds.bins[one], sum);
    has = has && !same;
    left &= ~lanes;
  }
  if (has) atomicAdd(&lds.bins[bin], w);
}
// One digit: the bin, from the top, in which the sum reaches `want`.  over: the sum above it, all: its own.
__device__ __forceinline__ unsigned draw_digit(DrawShared& lds, draw_u64 want, draw_u64& over, draw_u64& all) {
  constexpr int N = (1 << DRAW_DIGIT) / 1024;              // neighbouring bins a thread, from the top
  const int low = (1023 - (int)threadIdx.x) * N;
  draw_u64 bin[N], sum = 0, whole;
#pragma unroll
  for (int i = 0; i < N; ++i) { bin[i] = lds.bins[low + i]; sum += bin[i]; }
  draw_u64 before = over + draw_prefix(sum, lds.slots, whole);
  if (before < want && before + sum >= want) {
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      if (before < want && before + bin[i] >= want) { lds.found = (unsigned)(low + i); lds.found_sum = before; lds.found_all = bin[i]; }
      before += bin[i];
    }
  }
  __syncthreads();
  over = lds.found_sum; all = lds.found_all;
  return lds.found;                                        // written again behind the next digit's barriers
}
// The place of the first row, in the order of places, at which the sum of the rows' weights up to it reaches `want`; `over`: what lies
// above all rows that `each` goes through.  By digits of up to 12 bits of the keys' distance from the least one, so that the first digit
// spreads whatever the range (scores share their first bits: by those, most rows would meet at few addresses, one after the other),
// without the last bits that all keys share (16 of bf16's); then, where several rows share the border's key, of the ids.  All 1,024 threads
// call it; each(f) calls f(place, weight) for every row of the thread, weight() its weight, as often in all lanes of a wave (place 0: no
// row); of(key): a key's weight.  LISTS: a pass costs little (rows in LDS): the rows of a digit's bin, where they are few, go to the end at once.
template <bool LISTS, typename E, typename W>
__device__ __forceinline__ draw_u64 draw_border(DrawShared& lds, int rows, draw_u64 want, draw_u64 over, E each, W of) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned end[4] = {0, 0, 0, 0};                          // greatest key, greatest complement; all bits set somewhere, all clear somewhere
  each([&](draw_u64 place, auto) {
    const unsigned k = (unsigned)(place >> 32);
    if (place) { end[0] = max(end[0], k); end[1] = max(end[1], ~k); end[2] |= k; end[3] |= ~k; }
  });
  struct Or { __device__ __forceinline__ unsigned operator()(unsigned x, unsigned y) const { return x | y; } };
  end[0] = draw_wave_prefix(end[0], DrawMax()); end[1] = draw_wave_prefix(end[1], DrawMax());
  end[2] = draw_wave_prefix(end[2], Or()); end[3] = draw_wave_prefix(end[3], Or());
  __syncthreads();
  if (lane == 63) {
#pragma unroll
    for (int i = 0; i < 4; ++i) lds.ends[i][wave] = end[i];
  }
  __syncthreads();
  const unsigned hi = draw_lane(draw_row_prefix(lds.ends[0][lane & 15], DrawMax()), 15);
  unsigned base = ~draw_lane(draw_row_prefix(lds.ends[1][lane & 15], DrawMax()), 15);
  const unsigned differ = draw_lane(draw_row_prefix(lds.ends[2][lane & 15], Or()) & draw_row_prefix(lds.ends[3][lane & 15], Or()), 15);
  const int same = differ ? __builtin_ctz(differ) : 0;     // last bits that all share
  int left = hi > base ? 32 - __builtin_clz(hi - base) : same + 1;
  draw_u64 ties = 0;
  unsigned key = 0, upper = 0;
  // keys, then (upper != 0) the ids of the rows that have the key found: greater lower halves of places first
  while (true) {
    const int end_at = upper ? 0 : same, width = min(left - end_at, DRAW_DIGIT), shift = left - width;
    __syncthreads();
    for (int i = threadIdx.x; i < 1 << DRAW_DIGIT; i += 1024) lds.bins[i] = 0;
    if (threadIdx.x == 0) lds.listed = 0;
    __syncthreads();
    each([&](draw_u64 place, auto weight) {
      const unsigned k = upper ? (unsigned)place : (unsigned)(place >> 32);
      const bool has = place != 0 && (upper == 0 || (unsigned)(place >> 32) == upper) && k >= base && (draw_u64)(k - base) >> left == 0;
      draw_add(lds, has, (k - base) >> shift, has ? weight() : 0);
    });
    __syncthreads();
    base += draw_digit(lds, want, over, ties) << shift;
    left = shift;
    if (LISTS && !upper) {
      DrawShort& few = *reinterpret_cast<DrawShort*>(lds.bins);
      draw_u64* const list = lds.bins + (sizeof(DrawShort) + 7) / 8;
      each([&](draw_u64 place, auto) {
        const unsigned k = (unsigned)(place >> 32);
        if (place == 0 || k < base || (draw_u64)(k - base) >> left != 0) return;
        const unsigned n = atomicAdd(&lds.listed, 1u);
        if (n < DRAW_SHORT) list[n] = place;
      });
      __syncthreads();
      if (lds.listed <= DRAW_SHORT) return draw_border_short(few, lds.listed, want, over, [&](unsigned i) { return list[i]; }, of);          // uniform
    }
    if (left > end_at) continue;
    if (upper) return (draw_u64)upper << 32 | base;
    key = base;
    // all rows at the key are needed: no id decides
    if (want - over > ties - of(key)) return (draw_u64)key << 32;
    upper = key;
    base = ~(unsigned)(rows - 1);
    left = rows > 1 ? 32 - __builtin_clz((unsigned)(rows - 1)) : 1;
  }
}

// A key that the k greatest of the keys reach, and few others: the least of its bin among 1,024 from the least key to the greatest, again within
// the bin while that leaves a quarter too many.  All 1,024 threads call it; each(f) calls f(key) for every key of the thread (0: none), of
// which there are k at least.
template <typename E> __device__ __forceinline__ unsigned draw_bound(DrawShared& lds, unsigned k, E each) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned* bins = reinterpret_cast<unsigned*>(lds.bins);
  unsigned hi = 0, lo = 0, over = 0;                       // lo: of the keys' complements
  each([&](unsigned key) { if (key) { hi = max(hi, key); lo = max(lo, ~key); } });
  hi = draw_wave_prefix(hi, DrawMax());
  lo = draw_wave_prefix(lo, DrawMax());
  if (lane == 63) { lds.ends[0][wave] = hi; lds.ends[1][wave] = lo; }
  bins[threadIdx.x] = 0;
  __syncthreads();
  hi = draw_lane(draw_row_prefix(lds.ends[0][lane & 15], DrawMax()), 15);
  unsigned base = ~draw_lane(draw_row_prefix(lds.ends[1][lane & 15], DrawMax()), 15);
  int left = hi > base ? 32 - __builtin_clz(hi - base) : 1;
  while (true) {
    const int shift = max(left - 10, 0);
    each([&](unsigned key) { if (key >= base && (draw_u64)(key - base) >> left == 0) atomicAdd(&bins[(key - base) >> shift], 1u); });
    __syncthreads();
    const unsigned mine = bins[1023 - threadIdx.x];        // from the top
    unsigned all;
    const unsigned before = over + draw_prefix(mine, (unsigned*)lds.slots, all);
    bins[1023 - threadIdx.x] = 0;
    if (before < k && before + mine >= k) { lds.found = 1023 - threadIdx.x; lds.found_sum = before; lds.found_all = mine; }
    __syncthreads();
    base += lds.found << shift;
    over = (unsigned)lds.found_sum;
    left = shift;
    if (left == 0 || over + (unsigned)lds.found_all <= k + k / 4 + 8) return base;         // uniform
  }
}

// Chunks: as many as fill the device some eight times, of 2,048 to 2^21 rows.
struct DrawLayout { size_t stats, maxima, hist, range, totals, kept, listed, undone, lists, mass, bytes; int segments, chunks, chunk_rows, blocks, merge, groups, list, hist_bits, mass_pitch; };
static inline DrawLayout draw_layout(const mar_sampling* p) {
  DrawLayout L = {};
  if (p->num_rows <= DRAW_SMALL || p->num_queries == 0) { L.bytes = 256; return L; }
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  const size_t Q = (size_t)p->num_queries;
  L.segments = (int)((p->num_rows + DRAW_SEGMENT - 1) / DRAW_SEGMENT);
  int64_t chunks = 2048 / p->num_queries;
  if (chunks < (p->num_rows + (1 << 21) - 1) >> 21) chunks = (p->num_rows + (1 << 21) - 1) >> 21;
  chunks = chunks < 1 ? 1 : (chunks > 256 ? 256 : chunks);
  int64_t turns = (p->num_rows + 2048 * chunks - 1) / (2048 * chunks);
  L.chunk_rows = (int)(2048 * turns);
  L.chunks = (int)((p->num_rows + L.chunk_rows - 1) / L.chunk_rows);
  // Groups: some 4,096 to 8,192, which stay in registers where they are looked through, and enough for a top-k of up to 2,048; a chunk's turns by
  // blocks where there are too few, neighbouring threads merged where there are too many (5 x 1,000,003, top-k 50: 80 us with 62,720, 26 with
  // 7,840), up to 256 rows (1 x 20,000,000, top-k 1,000: 210 us with 312 rows, 273 with 2,496).  A large top-k has the groups that reach its bound looked through again, and wants them smaller: at most eight turns (100 x 1,000,003,
  // top-k 2,000: 248 -> 173 us), and twice as many as its rows, where there are so many turns.
  int64_t blocks = 4096 / (256 * L.chunks);
  if (p->top_k > 512) {
    const int64_t more = 16384 / (256 * L.chunks), eighth = more < turns / 8 ? more : turns / 8;
    const int64_t least = (2 * (p->top_k < DRAW_FEW ? p->top_k : DRAW_FEW) + 256 * L.chunks - 1) / (256 * L.chunks);
    blocks = blocks > eighth ? blocks : eighth;
    blocks = blocks > least ? blocks : least;
  }
  L.blocks = (int)(blocks < 1 ? 1 : (blocks > turns ? turns : blocks));
  L.merge = 1;
  const int64_t group_rows = 8 * ((turns + L.blocks - 1) / L.blocks);
  while (L.merge < 16 && 2 * L.merge * group_rows <= 256 && L.chunks * L.blocks * (256 / (2 * L.merge)) >= (p->top_k > 512 ? 16384 : 4096)) L.merge *= 2;
  L.groups = L.chunks * L.blocks * (256 / L.merge);
  // Of normal scores the border's range, a bin or two, holds up to 1 in 120 rows with bins as fine as they allow, more with 32 a binary order of
  // magnitude (rows far below all others): 1 / 58 over the deviation.  A workgroup holds 8,192 of them, the rest stays in memory (100 x 1,000,003,
  // deviation 0.67: 3.5 ms where all had to fit a workgroup, 0.29).
  L.list = (int)(p->num_rows / 32 < DRAW_LIST ? DRAW_LIST : p->num_rows / 32);
  L.stats = take(Q * L.chunks * sizeof(DrawChunk));
  L.maxima = take(Q * L.groups * 4);
  const size_t hists = Q * L.chunks * DRAW_BINS * 4, lists = Q * L.list * 8;
  L.hist = L.lists = take(hists > lists ? hists : lists);  // lists are written when the histograms have been read, by an earlier kernel
  L.hist_bits = 16;                                        // a bin's sum of a chunk stays below 2^32
  while ((int64_t)L.chunk_rows << L.hist_bits >= 1ll << 32) --L.hist_bits;
  L.range = take(Q * sizeof(DrawRange));
  L.totals = take(Q * L.chunks * 16);
  L.kept = take(Q * L.chunks * 4);
  L.listed = take(Q * 4);
  L.undone = take(Q * 4);
  L.mass_pitch = (L.segments + 15) / 16 * 16;              // lines of 128 bytes
  L.mass = take(Q * L.mass_pitch * 8);
  L.bytes = at;
  return L;
}
