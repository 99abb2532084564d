// Rows drawn from scores with temperature, top-k, top-p and min-p (gfx950).
//
// A row's place in the order (score descending, id ascending) is one number, so that every filter is a cut: rows whose place is not below it
// are kept.  Weights are integers W = round(2^n exp((s - max) / temperature)), n such that the sum of those that top-k leaves lies between
// 2^60 and 2^61 (which their sum in 32 bits says, whatever way a query goes): sums are exact in any order, and a border (top-p's, a draw's) falls
// where the integers say, whatever way found it.
//
// Up to 16,384 rows (k_draw_small): a workgroup a query holds them in registers (one query of 4,000 to 16,000 rows, no filter: 10 us; by the kernels
// below 18 to 20; 1,000 queries of 16,000 rows: 35 and 72).  More:
//   k_draw_scan    a workgroup a chunk: greatest score; sum of weights in fp32 where no histogram follows; maxima of groups of rows
//   k_draw_hist    queries without top-k, with top-p: weights by their binary order of magnitude, 1/32 apart
//   k_draw_range   the same queries: the bins that the border lies in, whatever the rounding
//   k_draw_weigh   queries without top-k: every row's integer weight: the sum of all, the sums of segments of 512 rows above the range, the
//                  range's rows by themselves
//   k_draw_rows    a workgroup a query.  Top-k: the k-th largest of the groups' maxima bounds the k-th best row from below; rows that reach it
//                  are picked from the groups whose maximum does, and everything else concerns those rows alone.  Others: the border among
//                  the range's rows, then the draws: the segment by the sums before it, the row by a wave that weighs it again
//   k_draw_slowly  what does not fit (borders among more rows than a list holds, top-k above 2,048) by digits over all rows
#include <type_traits>
#include "mar_sample_dev.h"

// ------------------------------------------------------------------------------------------ pieces -----
template <int TYPE> __device__ __forceinline__ void draw_nothing(const DrawArgs& a, int64_t q) {
  for (int d = threadIdx.x; d < a.draws; d += blockDim.x) {
    a.ids[q * a.draws + d] = -1;
    if (a.log_probs) a.log_probs[q * a.draws + d] = -__builtin_inff();
  }
  if (threadIdx.x == 0 && a.num_kept) a.num_kept[q] = 0;
}
__device__ __forceinline__ draw_u64 draw_target(float u, draw_u64 total) { return !(u > 0.f) ? 0 : (u >= 1.f ? total - 1 : draw_share_down(u, total)); }

// What the chunks of a query say together (all threads; up to 256 chunks).
struct DrawWhole { unsigned best; float sum; };
__device__ __forceinline__ DrawWhole draw_whole(const DrawArgs& a, int64_t q, float c, draw_u64* slots) {
  DrawWhole r = {0u, 0.f};
  DrawChunk mine = {0u, 0u, 0.f};
  if ((int)threadIdx.x < a.chunks) mine = a.stats[q * a.chunks + threadIdx.x];
  r.best = draw_reduce(mine.best, (unsigned*)slots, DrawMax());
  const float part = mine.best ? mine.sum * __builtin_amdgcn_exp2f(-draw_depth(draw_score(r.best), draw_score(mine.best), c)) : 0.f;
  r.sum = draw_sum(part, (float*)slots);
  return r;
}

// Bins to a binary order of magnitude: 32, doubled as long as all rows that weigh something beside the best fit, so that flat scores spread over the bins
// as well (100 x 1,000,003 in 16 bits, scores over the temperature of deviation 0.2: 3.4 ms for the call with 32, all of whose bins' rows no
// list holds, and 0.28).  Rows 63 binary orders below have no say, one or many (deviation 0.05 and one row at -1e9, which had 32 bins taken: 6.6
// ms and 0.29).
__device__ __forceinline__ float draw_fine(const DrawArgs& a, int64_t q, float c, unsigned best, draw_u64* slots) {
  unsigned low = 0;
  if ((int)threadIdx.x < a.chunks) {
    const DrawChunk s = a.stats[q * a.chunks + threadIdx.x];
    const float from = draw_score(best) - draw_window(c);
    if (s.low && draw_score(s.best) >= from) low = ~draw_key(fmaxf(draw_score(~s.low), from));
  }
  low = draw_reduce(low, (unsigned*)slots, DrawMax());
  const float depth = draw_depth(draw_score(best), draw_score(~low), c);
  float span = 63.f / 2, fine = 32.f;
  if (low) while (fine < 32768.f && depth <= span) { span /= 2; fine *= 2; }       // uniform
  return fine;
}

// The draws of a query: rows with place >= cut that score min-p's floor or more; mass: the segments' sums (LDS or memory), replaced by those before them.
template <int TYPE>
__device__ __forceinline__ void draw_rows(const DrawArgs& a, int64_t q, const DrawRow<TYPE>& row, const DrawWeights& w, draw_u64 cut, float floor, draw_u64* mass,
                                          draw_u64* slots) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, threads = blockDim.x;
  draw_u64 total = 0;
  for (int s0 = 0; s0 < a.segments; s0 += threads) {
    const int s = s0 + threadIdx.x;
    draw_u64 all;
    // past the CU's cache: sums in memory have been added to
    const draw_u64 m = s < a.segments ? __hip_atomic_load(&mass[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0, before = total + draw_prefix(m, slots, all);
    total += all;
    if (s < a.segments) mass[s] = before;
  }
  __syncthreads();
  const double log_total = w.log_sum(total);
  for (int d = wave; d < a.draws; d += threads >> 6) {     // a wave a draw
    draw_u64 target = draw_target(a.uniforms[q * a.draws + d], total);
    // the last segment that begins at or below the target, 64 at a time
    int from = 0, step = 1;
    while ((int64_t)step * 64 < a.segments) step *= 64;
    for (; step >= 1; step /= 64) {
      const int64_t s = from + (int64_t)lane * step;
      const bool below = s < a.segments && mass[s] <= target;
      from += (__popcll(__ballot(below)) - 1) * step;      // lane 0 is
    }
    target -= mass[from];
    const int64_t c = (int64_t)from * DRAW_SEGMENT + 8 * lane;
    unsigned key[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    if (c < a.rows) row.keys((int)c, key);
    draw_u64 each[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      each[e] = key[e] != 0 && draw_place(key[e], (unsigned)c + e) >= cut && draw_score(key[e]) >= floor ? w.of(key[e]) : 0;
      sum += each[e];
    }
    const draw_u64 run = draw_wave_prefix(sum), start = run - sum;
    if (start <= target && target < run) {                 // one lane
      int at = 0;
      unsigned k = key[0];
      draw_u64 upto = start + each[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) if (upto <= target) { upto += each[j]; at = j; k = key[j]; }
      a.ids[q * a.draws + d] = (int)c + at;
      if (a.log_probs) a.log_probs[q * a.draws + d] = w.log_prob(k, log_total);
    }
  }
}

// Up to 256 rows, with all that top-k (at least 1) leaves among them: four threads a row compare it with all others, once for the rank, which
// puts top-k's rows in order for their weights and sums, once for the place by id among those kept.  Called by 1,024 threads.
__device__ __forceinline__ void draw_short(const DrawArgs& a, int64_t q, DrawShort& lds, unsigned n, const DrawParams& par, unsigned best, double drop) {
  const unsigned tid = threadIdx.x, r = tid >> 2, part = tid & 3, padded = (n + 15) & ~15u;
  if (tid >= n && tid < padded) lds.row[tid].place = 0;    // comes after all others
  __syncthreads();
  draw_u64 mine = r < n ? lds.row[r].place : 0;
  // sums over the four threads of a row
  auto joined = [](auto v) { v += draw_moved<0xB1, 0xf>(v); return v + draw_moved<0x4E, 0xf>(v); };       // lanes 1 0 3 2, then 2 3 0 1
  unsigned rank = 0;
#pragma unroll 4
  for (unsigned i = part; i < padded; i += 4) rank += lds.row[i].place > mine;
  rank = joined(rank);
  const bool top = part == 0 && r < n && rank < (unsigned)par.top_k;
  const unsigned weighs = top ? draw_part(draw_score(best), (unsigned)(mine >> 32), draw_depth_scale(par)) : 0;
  const DrawWeights w = draw_weights(best, par, draw_parts(draw_sum(weighs, (unsigned*)lds.slots)));         // behind its barriers the rows have been read
  if (top) lds.row[rank].place = mine;
  __syncthreads();
  const unsigned m = min(n, (unsigned)par.top_k), padded_m = (m + 15) & ~15u;
  bool in = tid < m;                                       // a thread a row, by rank
  const draw_u64 place = in ? lds.row[tid].place : 0, weight = in ? w.of((unsigned)(place >> 32)) : 0;
  if (par.top_p < 2.f) {                                   // uniform
    draw_u64 sum;
    const draw_u64 before = draw_prefix(weight, lds.slots, sum), want = draw_share_up(par.top_p, sum);
    in = in && before < (want ? want : 1);
  }
  in = in && draw_score((unsigned)(place >> 32)) >= w.floor(drop);
  if (a.num_kept) {
    const unsigned kept = draw_sum(in ? 1u : 0u, (unsigned*)lds.slots);
    if (tid == 0) a.num_kept[q] = (int)kept;
  }
  const draw_u64 total = draw_sum(in ? weight : 0, lds.slots);
  const unsigned count = draw_sum(in && weight ? 1u : 0u, (unsigned*)lds.slots);
  if (tid < padded_m) lds.row[tid] = {in ? place : 0, in ? weight : 0};
  __syncthreads();
  // by id: places of lesser ids have greater lower halves
  mine = r < m ? lds.row[r].place : 0;
  const draw_u64 own = r < m ? lds.row[r].weight : 0;
  const unsigned id = ~(unsigned)mine;
  draw_u64 start = 0;
  unsigned at = 0;
#pragma unroll 4
  for (unsigned i = part; i < padded_m; i += 4) {
    const auto other = lds.row[i];
    const bool ahead = other.weight != 0 && ~(unsigned)other.place < id;
    at += ahead;
    start += ahead ? other.weight : 0;
  }
  at = joined(at);
  start = joined(start);
  if (own && part == 0) {
    lds.start[at] = start; lds.id[at] = id;
    lds.log_prob[at] = w.log_prob((unsigned)(mine >> 32), w.log_sum(total));
  }
  __syncthreads();
  for (int d = tid; d < a.draws; d += 1024) {
    const draw_u64 target = draw_target(a.uniforms[q * a.draws + d], total);
    unsigned from = 0;                                     // the last row that begins at or below the target
#pragma unroll
    for (unsigned step = DRAW_SHORT / 2; step >= 1; step /= 2) if (from + step < count && lds.start[from + step] <= target) from += step;
    a.ids[q * a.draws + d] = (int)lds.id[from];
    if (a.log_probs) a.log_probs[q * a.draws + d] = lds.log_prob[from];
  }
}

// Adds a row's weight to its bin, in units of 2^-bits of the bin's largest: 2^-(x / fine), x what the depth has below its bin's top;
// 1 - x l + (x l)^2 / 2, l = ln 2 / fine, is off by 2^-19 at most.  Rows that do not count, and those below 2^-63.9, go to 64 words
// behind the bins: additions to one address go one by one, and those would all meet at one (100 x 1,000,003 in 16 bits,
// a tenth of them counting: 509 us for the call at one, 251 at 64; all counting: 280 and 286).
struct DrawBins {
  float top, scale, w0, w1, w2;
  __device__ __forceinline__ DrawBins(float top, float c, float fine, int bits) : top(top), scale(c * fine), w0((float)(1 << bits)) {
    const float l = 0.69314718f / fine;
    w1 = -l * w0; w2 = 0.5f * l * l * w0;
  }
  __device__ __forceinline__ void operator()(unsigned* bins, float v) const {
    const float depth = __builtin_amdgcn_fmed3f((top - v) * scale, 0.f, DRAW_BINS - 1.f), x = __builtin_amdgcn_fractf(depth);
    atomicAdd(&bins[depth < DRAW_BINS - 1.f ? (int)depth : DRAW_BINS + (int)(threadIdx.x & 63)], (unsigned)__builtin_fmaf(x, __builtin_fmaf(x, w2, w1), w0));
  }
};
// The bins in which the border of top-p lies: thread t of 1,024 has the sums of bins 2 t and 2 t + 1.  A weight in the histogram is off by
// 2^-17 of itself at most by its depth (up to 64, in fp32) and polynomial and by a unit, 2^-bits at most of any; those left out are 2^-63.9
// of the best one each: so are sums.
__device__ __forceinline__ DrawRange draw_range(draw_u64 nx, draw_u64 ny, int bits, float fine, float top_p, draw_u64* slots, int* ends) {
  const int tid = threadIdx.x;
  if (tid == 0) { ends[0] = DRAW_BINS - 1; ends[1] = DRAW_BINS - 1; }
  const double x = (double)nx * exp2(-2 * tid / (double)fine), y = (double)ny * exp2(-(2 * tid + 1) / (double)fine);
  double all;
  const double before = draw_prefix(x + y, (double*)slots, all), off = __builtin_ldexp(2.0, -bits) + 0x1p-16, want = (double)top_p * all;
  // the first bin at whose end the border may have been reached, and the first at whose end it must have been
  const double may = want * (1.0 - off), must = want * (1.0 + off);
  if (before < may && before + x + y >= may) ends[0] = before + x >= may ? 2 * tid : 2 * tid + 1;
  if (before < must && before + x + y >= must) ends[1] = before + x >= must ? 2 * tid : 2 * tid + 1;
  __syncthreads();
  return {want <= 0.0 ? 0 : ends[0], want <= 0.0 ? 0 : ends[1], (float)__builtin_ldexp(all, -bits)};
}

// ------------------------------------------------------------------------------------------ up to 16,384 rows -----
// CUTS: some query may have top-k or top-p; without the code for them two workgroups fit a CU.  Top-k of up to 128 goes by the threads' maxima
// and a short list.  One query of 14,951 rows, top-k 50, top-p 0.95: 11.3 us; 1,000 queries, 100 draws each, no filter: 40 us, 15 million weights at 49
// instructions of the vector ALU each: bound by their issue.
template <int TYPE, bool CUTS>
__global__ void __launch_bounds__(1024, CUTS ? 4 : 8)
k_draw_small(DrawArgs a, int64_t first) {
  __shared__ union { DrawShared border; DrawShort list; draw_u64 before[2048]; } lds;
  __shared__ __attribute__((aligned(16))) union { float score[CUTS ? DRAW_SMALL : 4]; draw_u64 list[CUTS ? DRAW_LIST : 2]; } held;
  __shared__ draw_u64 slots[16];
  __shared__ draw_u64 starts[32];
  __shared__ unsigned listed, reached;
  __shared__ double drop;
  __shared__ int ends[2];
  const int64_t q = first + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const DrawRow<TYPE> row(a, q);
  const DrawParams par = draw_params(a, q);
  if (tid == 0) { listed = 0; reached = 0; }
  float v[2][8], mine = -__builtin_inff();                  // columns 8 tid .. and 8,192 + 8 tid ..: a wave holds segments `wave` and 16 + wave
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[b][e] = -__builtin_inff();
    if (8192 * b + 8 * tid < a.rows) row.scores_of(8192 * b + 8 * tid, v[b]);
  }
  if (wave == 0) drop = draw_drop(par);
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 8; ++e) mine = fmaxf(mine, v[b][e]);
  const unsigned best = draw_reduce(draw_key(mine), (unsigned*)slots, DrawMax());
  if (best == 0) { draw_nothing<TYPE>(a, q); return; }     // uniform
  auto place = [&](int b, int e) { return draw_place(draw_key(v[b][e]), (unsigned)(8192 * b + 8 * tid + e)); };
  draw_u64 cut = 1;
  if constexpr (CUTS) if (par.top_k > 0 && par.top_k <= 128 && par.top_k < a.rows) {       // uniform
    // the k-th largest of the threads' maxima bounds the k-th best row from below: few rows reach it
    const unsigned bound = draw_bound(lds.border, (unsigned)par.top_k, [&](auto f) { f(max(draw_key(mine), 1u)); });
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) if (draw_key(v[b][e]) >= bound) {
        const unsigned n = atomicAdd(&listed, 1u);
        if (n < DRAW_SHORT) lds.list.row[n].place = place(b, e);
      }
    __syncthreads();
    if (listed <= DRAW_SHORT) { draw_short(a, q, lds.list, listed, par, best, drop); return; }
  }
  const float c = draw_depth_scale(par), top = draw_score(best);
  DrawWeights w = {};
  bool found_cut = false;
  if constexpr (CUTS) if (par.top_p < 2.f && draw_all(a, par) && !draw_infinite(best)) {    // uniform
    // top-p alone: the border's range of bins by a histogram, then the border among the range's rows.  4,000 and 16,000 rows: 19 and 21 us a
    // query, 76 and 87 us 1,000 of them; by digits over all rows, as below, 35 and 47, 144 and 191
    unsigned* const bins = reinterpret_cast<unsigned*>(lds.border.bins);
    for (int i = tid; i < DRAW_BINS; i += 1024) bins[i] = 0;
    __syncthreads();
    const DrawBins add(top, c, 32.f, 17);                        // 2^14 rows in 32 bits
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) add(bins, v[b][e]);
    __syncthreads();
    const DrawRange range = draw_range(bins[2 * tid], bins[2 * tid + 1], 17, 32.f, par.top_p, slots, ends);
    w = draw_weights(best, par, range.sum);
    const float c32 = c * 32.f, low = (float)range.low, high = range.high < DRAW_BINS - 1 ? range.high + 1.f : __builtin_inff();
    draw_u64* const list = held.list;
    draw_u64 all = 0, above = 0, sum = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const draw_u64 x = w.of_score(v[b][e]);
        const float bin = (top - v[b][e]) * c32;
        all += x;
        above += bin < low ? x : 0;
        if (bin >= low && bin < high) {
          sum += x;
          const unsigned n = atomicAdd(&listed, 1u);
          if (n < DRAW_LIST) list[n] = place(b, e);
        }
      }
    all = draw_sum(all, slots); above = draw_sum(above, slots); sum = draw_sum(sum, slots);           // their barriers order the list
    draw_u64 want = draw_share_up(par.top_p, all);
    if (want == 0) want = 1;
    const unsigned n = listed;
    // else many equal rows, or temperatures whose inverse 32 bits do not hold
    found_cut = n <= DRAW_LIST && above < want && above + sum >= want;
    if (found_cut && n <= DRAW_SHORT) cut = draw_border_short(lds.list, n, want, above, [&](unsigned i) { return list[i]; }, [&](unsigned k) { return w.of(k); });
    else if (found_cut) cut = draw_border<true>(lds.border, a.rows, want, above, [&](auto f) {
      for (unsigned i = tid; i - tid < n; i += 1024) { const draw_u64 p = i < n ? list[i] : 0; f(p, [&] { return w.of((unsigned)(p >> 32)); }); }
    }, [&](unsigned k) { return w.of(k); });
  }
  bool ranks = false;                                      // top-k leaves rows out
  if constexpr (CUTS) if (par.top_k > 0 && par.top_k < a.rows) {       // uniform
    unsigned count = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) count += v[b][e] > -__builtin_inff();
    ranks = (unsigned)par.top_k < draw_sum(count, (unsigned*)slots);
    // larger top-k: a bound among all rows, and everything else concerns the rows that reach it (16,000 rows, top-k 1,000, top-p 0.9: 28 us; by
    // digits over all rows, as below, 53; 1,000 queries: 114 and 218)
    if (ranks) {
      const unsigned k = (unsigned)par.top_k;
      const unsigned bound = draw_bound(lds.border, k, [&](auto f) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 8; ++e) f(draw_key(v[b][e]));
      });
      unsigned here = 0;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 8; ++e) here += draw_key(v[b][e]) >= bound;
      const unsigned upto = draw_wave_prefix(here);
      unsigned at = 0;
      if (lane == 63 && upto) at = atomicAdd(&reached, upto);
      at = draw_lane(at, 63) + upto - here;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 8; ++e) if (draw_key(v[b][e]) >= bound) { if (at < DRAW_LIST) held.list[at] = place(b, e); ++at; }
      __syncthreads();
      const unsigned n = reached;
      found_cut = n <= DRAW_LIST;                          // else many equal rows
      if (found_cut) {
        auto each = [&](auto f) { for (unsigned i = tid; i - tid < n; i += 1024) f(i < n ? held.list[i] : 0); };
        cut = (draw_u64)bound << 32;
        for (int kind = k < n ? 0 : 1; kind < 2; ++kind) { // by counts, then by weights
          draw_u64 want = k;
          const draw_u64 last = cut;
          if (kind == 1) {
            unsigned parts = 0;
            each([&](draw_u64 p) { parts += p >= last ? draw_part(top, (unsigned)(p >> 32), c) : 0; });
            w = draw_weights(best, par, draw_parts(draw_sum(parts, (unsigned*)slots)));
            if (par.top_p >= 2.f) break;
            draw_u64 sum = 0;
            each([&](draw_u64 p) { sum += p >= last ? w.of((unsigned)(p >> 32)) : 0; });
            want = draw_share_up(par.top_p, draw_sum(sum, slots));
            if (want == 0) want = 1;
          }
          cut = draw_border<true>(lds.border, a.rows, want, 0, [&](auto f) {
            each([&](draw_u64 p) { f(p >= last ? p : 0, [&] { return kind == 1 ? w.of((unsigned)(p >> 32)) : draw_one(); }); });
          }, [&](unsigned key) { return kind == 1 ? w.of(key) : draw_one(); });
        }
      }
    }
  }
  if (!found_cut && !ranks) {
    float approx = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) approx += __builtin_amdgcn_exp2f(-draw_depth(top, v[b][e], c));
    w = draw_weights(best, par, draw_sum(approx, (float*)slots));
  }
  if constexpr (CUTS) if (!found_cut && (ranks || par.top_p < 2.f)) {       // uniform
    // through LDS: loops over the rows take a sixteenth of the code, and no registers beside the weights'
    struct Eight { float v[8]; };
#pragma unroll
    for (int b = 0; b < 2; ++b) *reinterpret_cast<Eight*>(held.score + 8192 * b + 8 * tid) = __builtin_bit_cast(Eight, v[b]);
    __syncthreads();
    auto each = [&](auto f) {
#pragma unroll 2
      for (int i = tid; i < DRAW_SMALL; i += 1024) f(draw_place(draw_key(held.score[i]), (unsigned)i));
    };
    if (ranks) {
      cut = draw_border<true>(lds.border, a.rows, (draw_u64)par.top_k, 0, [&](auto f) { each([&](draw_u64 place) { f(place, draw_one); }); },
                              [](unsigned) { return draw_one(); });
      float approx = 0.f;
      each([&](draw_u64 place) { approx += place >= cut ? __builtin_amdgcn_exp2f(-draw_depth(top, draw_score((unsigned)(place >> 32)), c)) : 0.f; });
      w = draw_weights(best, par, draw_sum(approx, (float*)slots));
    }
    if (par.top_p < 2.f) {
      draw_u64 all = 0;
      const draw_u64 top_k = cut;
      each([&](draw_u64 place) { all += place >= top_k ? w.of((unsigned)(place >> 32)) : 0; });
      const draw_u64 want = draw_share_up(par.top_p, draw_sum(all, slots));
      cut = draw_border<true>(lds.border, a.rows, want ? want : 1, 0, [&](auto f) { each([&](draw_u64 place) { f(place >= top_k ? place : 0, [&] { return w.of((unsigned)(place >> 32)); }); }); },
                               [&](unsigned k) { return w.of(k); });
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const Eight back = *reinterpret_cast<const Eight*>(held.score + 8192 * b + 8 * tid);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[b][e] = back.v[e];
    }
  }
  const float floor = w.floor(drop);
  unsigned kept = 0;
  draw_u64 sum[2] = {0, 0}, run[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const draw_u64 x = w.of_score(v[b][e]);
      const bool in = (CUTS ? place(b, e) >= cut : v[b][e] > -__builtin_inff()) && v[b][e] >= floor;
      kept += in;
      sum[b] += in ? x : 0;
    }
    run[b] = draw_wave_prefix(sum[b]);
  }
  if (a.num_kept) {                                        // uniform
    kept = draw_sum(kept, (unsigned*)slots);
    if (tid == 0) a.num_kept[q] = (int)kept;
  }
  __syncthreads();                                         // `before` takes the place of the borders' LDS
#pragma unroll
  for (int b = 0; b < 2; ++b) if (lane == 63) starts[16 * b + wave] = run[b];
  __syncthreads();
  const draw_u64 m = lane < 32 ? starts[lane] : 0, upto = draw_wave_prefix(m), total = draw_lane(upto, 31);      // every wave for itself
#pragma unroll
  for (int b = 0; b < 2; ++b) lds.before[1024 * b + tid] = draw_lane(upto - m, 16 * b + wave) + run[b] - sum[b];
  __syncthreads();
  // a thread a draw: the eight columns by the sums before them, the row by weighing those again
  const double log_total = w.log_sum(total);
  for (int d = tid; d < a.draws; d += 1024) {
    const draw_u64 target = draw_target(a.uniforms[q * a.draws + d], total);
    int at = 0;                                            // the last that begin at or below the target
#pragma unroll
    for (int step = 1024; step >= 1; step /= 2) if (lds.before[at + step] <= target) at += step;        // at + step < 2,048
    float score[8], found = 0.f;
    row.scores_of(8 * at, score);
    draw_u64 sum = lds.before[at];
    int column = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const draw_u64 x = w.of_score(score[e]);
      const bool in = (CUTS ? draw_place(draw_key(score[e]), (unsigned)(8 * at + e)) >= cut : score[e] > -__builtin_inff()) && score[e] >= floor;
      sum += in ? x : 0;
      if (column < 0 && sum > target) { column = e; found = score[e]; }
    }
    a.ids[q * a.draws + d] = 8 * at + column;
    if (a.log_probs) a.log_probs[q * a.draws + d] = w.log_prob(draw_key(found), log_total);
  }
}

// ------------------------------------------------------------------------------------------ more rows -----
// A workgroup a chunk of a query.  Group (chunk, block b, i): the columns of threads merge i .. merge i + merge - 1 in the iterations of block b.  Bound by memory: 100 x
// 1,000,003 bf16: 38 us, 5.3 TB/s (part of the scores comes out of the last-level cache); 64 x 131,072 fp32: 7 to 10 us.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_draw_scan(DrawArgs a, int64_t first) {
  __shared__ draw_u64 slots[16];
  const int64_t unit = first + blockIdx.x, q = unit / a.chunks;
  const int chunk = (int)(unit - q * a.chunks), tid = threadIdx.x;
  const DrawRow<TYPE> row(a, q);
  const DrawParams par = draw_params(a, q);
  const bool few = draw_few(a, par);
  const float c = draw_depth_scale(par);
  const int begin = chunk * a.chunk_rows, end = (int)min((int64_t)a.rows, (int64_t)begin + a.chunk_rows);
  const int turns = a.chunk_rows / 2048, turns_block = (turns + a.blocks - 1) / a.blocks;
  const bool sums = !few && draw_all(a, par) && par.top_p >= 2.f;
  const bool lows = !few && draw_all(a, par) && par.top_p < 2.f;
  float best = -__builtin_inff(), low = __builtin_inff(), sum = 0.f, group = best;
  const float window = draw_window(c);
  const int width = 256 / a.merge;
  unsigned* maxima = a.maxima + q * a.groups + (int64_t)chunk * a.blocks * width + tid / a.merge;
  const bool first_of = tid % a.merge == 0;
  int block = 0, left = turns_block;
  for (int i = 0; i < turns; ++i) {
    const int64_t at = (int64_t)begin + i * 2048 + 8 * tid;
    if (at < end) {
      float v[8], here = -__builtin_inff();
      row.raw((int)at, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) here = fmaxf(here, v[e]);          // NaN gives way
      here = fminf(here, DRAW_TOP);
      group = fmaxf(group, here);
      if (lows) {                                          // uniform
        // of rows within the window of the best so far; where that leaves it behind what came before is forgotten, or ends at its edge
        const float from = fmaxf(best, here) - window;
        float least = DRAW_TOP;
#pragma unroll
        for (int e = 0; e < 8; ++e) least = fminf(least, v[e]);
        if (!(least > -__builtin_inff() && least >= from)) {       // some do not count, or weigh nothing
          least = __builtin_inff();
#pragma unroll
          for (int e = 0; e < 8; ++e) least = fminf(least, v[e] > -__builtin_inff() && v[e] >= from ? v[e] : __builtin_inff());
        }
        low = fminf(best >= from ? fmaxf(low, from) : __builtin_inff(), least);
      }
      if (sums) {
        if (here > best) sum = sum > 0.f ? sum * __builtin_amdgcn_exp2f(-draw_depth(here, best, c)) : 0.f;
        const float top = fmaxf(best, here);
        if (top > -__builtin_inff()) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sum += __builtin_amdgcn_exp2f(-draw_depth(top, fminf(fmaxf(v[e], -DRAW_TOP), top), c));
        }
      }
      best = fmaxf(best, here);
    }
    if (--left == 0 || i + 1 == turns) {
      if (few) {                                           // uniform
        for (int i = 1; i < a.merge; i *= 2) group = fmaxf(group, __shfl_xor(group, i));
        if (first_of) maxima[width * block] = draw_key(group);
      }
      group = -__builtin_inff(); ++block; left = turns_block;
    }
  }
  if (few && first_of) for (; block < a.blocks; ++block) maxima[width * block] = 0;
  const unsigned mine = draw_key(best), all = draw_reduce(mine, (unsigned*)slots, DrawMax());
  sum = mine ? sum * __builtin_amdgcn_exp2f(-draw_depth(draw_score(all), best, c)) : 0.f;
  sum = draw_sum(sum, (float*)slots);
  unsigned least = 0;
  if (lows && all) {                                       // uniform
    const float from = draw_score(all) - window;
    least = draw_reduce(mine && best >= from ? ~draw_key(fmaxf(low, from)) : 0u, (unsigned*)slots, DrawMax());
  }
  if (tid == 0) {
    a.stats[q * a.chunks + chunk] = {all, least, sum};
    if (chunk == 0) a.listed[q] = 0;
  }
}

// Other queries with top-p: a chunk's weights by their bins.  20 instructions and an addition in LDS an element: 100 x 1,000,003: 58 us, bound
// by those.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_draw_hist(DrawArgs a, int64_t first) {
  __shared__ unsigned bins[DRAW_BINS + 64];
  __shared__ draw_u64 slots[16];
  const int64_t unit = first + blockIdx.x, q = unit / a.chunks;
  const int chunk = (int)(unit - q * a.chunks), tid = threadIdx.x;
  const DrawParams par = draw_params(a, q);
  if (draw_few(a, par) || !draw_all(a, par) || par.top_p >= 2.f) return;
  const DrawRow<TYPE> row(a, q);
  const float c = draw_depth_scale(par);
  for (int i = tid; i < DRAW_BINS; i += 256) bins[i] = 0;
  const DrawWhole whole = draw_whole(a, q, c, slots);
  if (draw_infinite(whole.best)) return;
  const DrawBins add(draw_score(whole.best), c, draw_fine(a, q, c, whole.best, slots), a.hist_bits);
  const int begin = chunk * a.chunk_rows, end = (int)min((int64_t)a.rows, (int64_t)begin + a.chunk_rows);
  for (int64_t at = (int64_t)begin + 8 * tid; at < end; at += 2048) {
    float v[8];
    row.raw((int)at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) add(bins, fmaxf(v[e], -__builtin_inff()));         // NaN gives way
  }
  __syncthreads();
  unsigned* out = a.hist + unit * DRAW_BINS;
  for (int i = tid; i < DRAW_BINS; i += 256) out[i] = bins[i];
}

// A workgroup a query: 20 to 256 chunks' bins of 8 KB each, read by one CU: 7 to 8 us.
__global__ void __launch_bounds__(1024)
k_draw_range(DrawArgs a, int64_t first) {
  __shared__ draw_u64 slots[16];
  __shared__ int ends[2];
  const int64_t q = first + blockIdx.x;
  const DrawParams par = draw_params(a, q);
  const int tid = threadIdx.x;
  if (draw_few(a, par) || !draw_all(a, par)) return;
  if (par.top_p >= 2.f) return;
  draw_u64 nx = 0, ny = 0;                                 // bins 2 tid and 2 tid + 1
#pragma unroll 8
  for (int k = 0; k < a.chunks; ++k) {
    const uint2 v = *reinterpret_cast<const uint2*>(a.hist + (q * a.chunks + k) * DRAW_BINS + 2 * tid);
    nx += v.x; ny += v.y;
  }
  const float c = draw_depth_scale(par), fine = draw_fine(a, q, c, draw_whole(a, q, c, slots).best, slots);
  const DrawRange range = draw_range(nx, ny, a.hist_bits, fine, par.top_p, slots, ends);
  if (tid == 0) a.range[q] = range;
}

// Integer weights of a chunk.  Bound by the issue of vector instructions: 50 a weight, of which 10 are the polynomial's; 100 x 1,000,003: 159 us.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_draw_weigh(DrawArgs a, int64_t first) {
  __shared__ draw_u64 slots[16], list[DRAW_LIST_CHUNK];
  __shared__ unsigned listed, list_at;
  __shared__ double drop;
  const int64_t unit = first + blockIdx.x, q = unit / a.chunks;
  const int chunk = (int)(unit - q * a.chunks), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) listed = 0;
  const DrawParams par = draw_params(a, q);
  if (draw_few(a, par) || !draw_all(a, par)) return;
  if (wave == 0) drop = draw_drop(par);
  const DrawRow<TYPE> row(a, q);
  const float c = draw_depth_scale(par);
  const DrawWhole whole = draw_whole(a, q, c, slots);
  if (whole.best == 0 || draw_infinite(whole.best)) return;
  const DrawRange range = par.top_p < 2.f ? a.range[q] : DrawRange{0, 0, 0.f};
  const DrawWeights w = draw_weights(whole.best, par, par.top_p < 2.f ? range.sum : whole.sum);
  const float floor = w.floor(drop);
  // bins by their depth, as the histogram counts them
  const float top = draw_score(whole.best), scale = par.top_p < 2.f ? c * draw_fine(a, q, c, whole.best, slots) : 0.f, low = (float)range.low, high = range.high < DRAW_BINS - 1 ? range.high + 1.f : __builtin_inff();
  const int begin = chunk * a.chunk_rows, end = (int)min((int64_t)a.rows, (int64_t)begin + a.chunk_rows);
  draw_u64 all = 0, above = 0;
  unsigned kept = 0;
  auto segments = [&](auto cuts, auto floors) {            // with top-p; with min-p
    constexpr bool CUTS = decltype(cuts)::value, FLOOR = decltype(floors)::value;
    for (int64_t s = (int64_t)begin + wave * DRAW_SEGMENT; s < end; s += 4 * DRAW_SEGMENT) {
      const int64_t at = s + 8 * lane;
      draw_u64 sum = 0;
      if (at < end) {
        float v[8];
        row.raw((int)at, v);
        draw_u64 near[8];                                  // lanes whose row lies in the range
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const draw_u64 x = w.of_score(v[e]);
          bool in = CUTS || v[e] > -__builtin_inff();      // a row that does not count lies below every range
          if (CUTS) {
            const float bin = (top - v[e]) * scale;
            in = bin < low;
            all += x;
            near[e] = __builtin_amdgcn_ballot_w64(bin >= low) & __builtin_amdgcn_ballot_w64(bin < high);
            if (FLOOR) above += in ? x : 0;                // before min-p: top-p goes by it
          }
          if (FLOOR) in = in && v[e] >= floor;
          sum += in ? x : 0;
          kept += in;
        }
        if (CUTS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) if (near[e]) {       // uniform
            const float bin = (top - v[e]) * scale;
            if (!(bin >= low && bin < high)) continue;
            const unsigned n = atomicAdd(&listed, 1u);
            const draw_u64 place = draw_place(draw_key(v[e]), (unsigned)at + e);
            if (n < DRAW_LIST_CHUNK) list[n] = place;
            else if (const unsigned m = atomicAdd(&a.listed[q], 1u); m < (unsigned)a.list) a.lists[q * a.list + m] = place;
          }
          if (!FLOOR) above += sum;
        }
      }
      sum = draw_wave_sum(sum);
      if (lane == 0) a.mass[q * a.mass_pitch + s / DRAW_SEGMENT] = sum;
    }
  };
  const std::true_type yes; const std::false_type no;
  if (par.top_p < 2.f) { if (par.min_p > 0.f) segments(yes, yes); else segments(yes, no); }
  else { if (par.min_p > 0.f) segments(no, yes); else segments(no, no); }
  all = draw_sum(all, slots);
  above = draw_sum(above, slots);
  kept = draw_sum(kept, (unsigned*)slots);
  const unsigned n = min(listed, (unsigned)DRAW_LIST_CHUNK);          // the reductions' barriers lie behind the last one
  if (threadIdx.x == 0) {
    a.totals[2 * unit] = all; a.totals[2 * unit + 1] = above;
    a.kept[unit] = kept;
    list_at = n ? atomicAdd(&a.listed[q], n) : 0;
  }
  if (n == 0) return;                                      // uniform
  __syncthreads();
  for (unsigned i = threadIdx.x; i < n; i += 256) if (list_at + i < (unsigned)a.list) a.lists[q * a.list + list_at + i] = list[i];
}

// A workgroup a query.  A chain of short steps with barriers between them, bound by their latency: 64 queries of 131,072 rows: without filters
// 9 us, top-k 50: 14, top-k 300: 20, top-k 1,000 and top-p 0.9: 32, top-p alone: 15; 100 of 1,000,003, top-p alone: 27.
template <int TYPE>
__global__ void __launch_bounds__(1024)
k_draw_rows(DrawArgs a, int64_t first) {
  __shared__ union { DrawShared border; DrawShort few; } lds;
  __shared__ draw_u64 list[DRAW_LIST];
  __shared__ union { unsigned groups[2 * DRAW_FEW]; draw_u64 mass[2048]; } near;
  __shared__ unsigned listed, grouped;
  __shared__ double drop;
  const int64_t q = first + blockIdx.x;
  const DrawParams par = draw_params(a, q);
  const int tid = threadIdx.x;
  if (tid == 0) { listed = 0; grouped = 0; }
  if (tid < 64) drop = draw_drop(par);
  const DrawRow<TYPE> row(a, q);
  const DrawWhole whole = draw_whole(a, q, draw_depth_scale(par), lds.border.slots);
  if (tid == 0) a.undone[q] = 0;
  if (whole.best == 0) { draw_nothing<TYPE>(a, q); return; }         // uniform, like all conditions that end in a return or a barrier
  const bool few = draw_few(a, par), cuts = par.top_p < 2.f;
  DrawWeights w = draw_weights(whole.best, par, draw_all(a, par) && cuts ? a.range[q].sum : whole.sum);       // few: anew
  const bool held = a.segments <= 2048;                    // the segments' sums fit LDS
  draw_u64* mass = held ? near.mass : a.mass + q * a.mass_pitch;
  draw_u64 cut = 1, all = 0, above = 0;                    // of the listed rows; sums of weights: of all rows for top-p, of those above the list
  unsigned n, kept = 0;
  bool slowly;
  if (few) {
    const unsigned* maxima = a.maxima + q * a.groups;
    unsigned some[8];                                      // the first 8,192 maxima stay in registers
#pragma unroll
    for (int i = 0; i < 8; ++i) some[i] = tid + 1024 * i < a.groups ? maxima[tid + 1024 * i] : 0;
    auto groups = [&](auto f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) if (1024 * i < a.groups) f(some[i], tid + 1024 * i);
      for (int g = tid + 8192; g - tid < a.groups; g += 1024) f(g < a.groups ? maxima[g] : 0, g);
    };
    // the k-th largest maximum, or somewhat less: k rows at least reach it
    const unsigned bound = draw_bound(lds.border, (unsigned)par.top_k, [&](auto f) { groups([&](unsigned m, int g) { f(g < a.groups ? max(m, 1u) : 0u); }); });
    groups([&](unsigned m, int g) {
      if (m < bound) return;
      const unsigned at = atomicAdd(&grouped, 1u);
      if (at < 2 * DRAW_FEW) near.groups[at] = (unsigned)g;
    });
    __syncthreads();
    const unsigned found = grouped;
    if (found <= 2 * DRAW_FEW) {
      // a group's turns and threads are work for a thread each
      const int turns = a.chunk_rows / 2048, turns_block = (turns + a.blocks - 1) / a.blocks, width = 256 / a.merge, per_chunk = a.blocks * width;
      const unsigned each = (unsigned)(turns_block * a.merge), items = found * each;
      for (unsigned i0 = 0; i0 < items; i0 += 4 * 1024) {  // four a thread on their way
        unsigned key[4][8];
        int column[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned i = i0 + 1024 * j + tid;
          column[j] = -1;
          if (i < items) {
            const int g = (int)near.groups[i / each], chunk = g / per_chunk, block = (g - chunk * per_chunk) / width, part = (int)(i % each);
            const int turn = block * turns_block + part / a.merge;
            const int64_t c = (int64_t)chunk * a.chunk_rows + turn * 2048 + 8 * (g % width * a.merge + part % a.merge);
            if (turn < turns && c < min((int64_t)a.rows, (int64_t)(chunk + 1) * a.chunk_rows)) { column[j] = (int)c; row.keys((int)c, key[j]); }
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (i0 + 1024 * j >= items) break;               // uniform
          unsigned here = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) here += column[j] >= 0 && key[j][e] >= bound;
          const unsigned upto = draw_wave_prefix(here);
          unsigned at = 0;
          if ((tid & 63) == 63 && upto) at = atomicAdd(&listed, upto);
          at = draw_lane(at, 63) + upto - here;
          if (here) {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (key[j][e] >= bound) { if (at < DRAW_LIST) list[at] = draw_place(key[j][e], (unsigned)column[j] + e); ++at; }
          }
        }
      }
    }
    __syncthreads();
    n = listed;
    slowly = found > 2 * DRAW_FEW || n > DRAW_LIST;        // many equal rows
    cut = (draw_u64)bound << 32;
    if (!slowly && n <= DRAW_SHORT) {
      if (tid < (int)n) lds.few.row[tid].place = list[tid];
      __syncthreads();
      draw_short(a, q, lds.few, n, par, whole.best, drop);
      return;
    }
    if (!slowly) for (int s = tid; s < a.segments; s += 1024) mass[s] = 0;
  } else {
    n = cuts ? a.listed[q] : 0;
    slowly = !draw_all(a, par) || draw_infinite(whole.best) || n > (unsigned)a.list;
    if (!slowly) {
      if (n <= DRAW_LIST) for (unsigned i = tid; i < n; i += 1024) list[i] = a.lists[q * a.list + i];
      if (held) {
#pragma unroll
        for (int i = 0; i < 2; ++i) if (tid + 1024 * i < a.segments) near.mass[tid + 1024 * i] = a.mass[q * a.mass_pitch + tid + 1024 * i];
      }
      if (tid < a.chunks) {
        all = a.totals[2 * (q * a.chunks + tid)]; above = a.totals[2 * (q * a.chunks + tid) + 1];
        kept = a.kept[q * a.chunks + tid];
      }
      all = draw_sum(all, lds.border.slots);
      above = draw_sum(above, lds.border.slots);
    }
  }
  if (!slowly) {
    __syncthreads();
    const draw_u64* const far = a.lists + q * a.list;         // where the workgroup does not hold them
    auto each = [&](auto f) { for (unsigned i = tid; i - tid < n; i += 1024) f(i < n ? (n <= DRAW_LIST ? list[i] : far[i]) : 0); };
    // top-k by counts, then top-p by weights
    for (int kind = few && (unsigned)par.top_k < n ? 0 : 1; kind < 2; ++kind) {
      draw_u64 want = (draw_u64)par.top_k;
      const draw_u64 last = cut;
      if (kind == 1) {
        if (few) {
          const float top = draw_score(whole.best), c = draw_depth_scale(par);
          unsigned parts = 0;
          each([&](draw_u64 place) { parts += place >= last && place ? draw_part(top, (unsigned)(place >> 32), c) : 0; });
          w = draw_weights(whole.best, par, draw_parts(draw_sum(parts, (unsigned*)lds.border.slots)));
        }
        if (!cuts) break;
        draw_u64 sum = 0;
        each([&](draw_u64 place) { sum += place >= last ? w.of((unsigned)(place >> 32)) : 0; });
        sum = draw_sum(sum, lds.border.slots);
        want = draw_share_up(par.top_p, few ? sum : all);
        if (want == 0) want = 1;
        // temperatures whose inverse 32 bits do not hold: the histogram was of something else
        slowly = above >= want || above + sum < want;
      }
      if (slowly) break;
      if (n <= DRAW_SHORT) {                               // of top-p: top-k's few rows went another way
        __syncthreads();                                   // all have their sums
        cut = draw_border_short(lds.few, n, want, above, [&](unsigned i) { return list[i]; }, [&](unsigned k) { return w.of(k); });
      } else cut = draw_border<true>(lds.border, a.rows, want, kind == 1 ? above : 0, [&](auto f) {
        each([&](draw_u64 place) { f(place >= last ? place : 0, [&] { return kind == 1 ? w.of((unsigned)(place >> 32)) : draw_one(); }); });
      }, [&](unsigned k) { return kind == 1 ? w.of(k) : draw_one(); });
    }
    if (!slowly) {
      const float floor = w.floor(drop);
      each([&](draw_u64 place) {
        if (place < cut) return;
        if (draw_score((unsigned)(place >> 32)) < floor) return;
        const draw_u64 x = w.of((unsigned)(place >> 32));
        ++kept;
        if (x) atomicAdd(&mass[~(unsigned)place / DRAW_SEGMENT], x);
      });
      kept = draw_sum(kept, (unsigned*)lds.border.slots);
      if (tid == 0 && a.num_kept) a.num_kept[q] = (int)kept;
      __syncthreads();
      draw_rows<TYPE>(a, q, row, w, cut, floor, mass, lds.border.slots);
    }
  }
  if (tid == 0) a.undone[q] = slowly;
}

// Queries that the kernel before could not do: everything by digits over all rows.  A kernel of its own: with this code in the other one,
// that took 10 to 15 us longer for all queries.  4 us where there are none.
template <int TYPE>
__global__ void __launch_bounds__(1024)
k_draw_slowly(DrawArgs a, int64_t first) {
  __shared__ DrawShared lds;
  const int64_t q = first + blockIdx.x;
  if (!a.undone[q]) return;                                // uniform
  const DrawRow<TYPE> row(a, q);
  const DrawParams par = draw_params(a, q);
  const unsigned best = draw_whole(a, q, 0.f, lds.slots).best;
  draw_u64* mass = a.mass + q * a.mass_pitch;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto each = [&](auto f) {
    for (int64_t c0 = 0; c0 < a.rows; c0 += 8 * 1024) {
      const int64_t c = c0 + 8 * tid;
      unsigned key[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
      if (c < a.rows) row.keys((int)c, key);
#pragma unroll
      for (int e = 0; e < 8; ++e) f(draw_place(key[e], (unsigned)c + e));
    }
  };
  auto ones = [&](auto f) { each([&](draw_u64 place) { f(place, draw_one); }); };
  const float top = draw_score(best), c = draw_depth_scale(par);
  draw_u64 cut = 1;
  unsigned count = 0;
  if (par.top_k > 0) { each([&](draw_u64 place) { count += place != 0; }); count = draw_sum(count, (unsigned*)lds.slots); }
  if (par.top_k > 0 && (unsigned)par.top_k < count) cut = draw_border<false>(lds, a.rows, (draw_u64)par.top_k, 0, ones, [](unsigned) { return draw_one(); });
  float approx = 0.f;
  each([&](draw_u64 place) { if (place >= cut) approx += __builtin_amdgcn_exp2f(-draw_depth(top, draw_score((unsigned)(place >> 32)), c)); });
  const DrawWeights w = draw_weights(best, par, draw_sum(approx, (float*)lds.slots));
  if (par.top_p < 2.f) {
    draw_u64 all = 0;
    each([&](draw_u64 place) { if (place >= cut) all += w.of((unsigned)(place >> 32)); });
    all = draw_sum(all, lds.slots);
    const draw_u64 want = draw_share_up(par.top_p, all), top_k = cut;
    // rows below top-k's cut have no say: they come after the border
    cut = draw_border<false>(lds, a.rows, want ? want : 1, 0, [&](auto f) { each([&](draw_u64 place) { f(place >= top_k ? place : 0, [&] { return w.of((unsigned)(place >> 32)); }); }); },
                      [&](unsigned k) { return w.of(k); });
  }
  const float floor = w.floor(draw_drop(par));
  unsigned kept = 0;
  for (int s = wave; s < a.segments; s += 16) {
    const int64_t c = (int64_t)s * DRAW_SEGMENT + 8 * lane;
    draw_u64 sum = 0;
    if (c < a.rows) {
      unsigned key[8];
      row.keys((int)c, key);
#pragma unroll
      for (int e = 0; e < 8; ++e) if (key[e] && draw_place(key[e], (unsigned)c + e) >= cut && draw_score(key[e]) >= floor) { sum += w.of(key[e]); ++kept; }
    }
    sum = draw_wave_sum(sum);
    if (lane == 0) mass[s] = sum;
  }
  kept = draw_sum(kept, (unsigned*)lds.slots);
  if (tid == 0 && a.num_kept) a.num_kept[q] = (int)kept;
  __syncthreads();
  draw_rows<TYPE>(a, q, row, w, cut, floor, mass, lds.slots);
}

// ------------------------------------------------------------------------------------------ launches -----
// Kernels that no query of the call can need, as far as the host knows, are left out.
template <int TYPE> static void launch_draws(const DrawArgs& a, int64_t queries, hipStream_t st) {
  if (a.rows <= DRAW_SMALL) {
    const bool cuts = a.temperatures || a.temperature == 0.f || a.top_ks || a.top_k > 0 || a.top_ps || a.top_p < 1.f;
    sm_launches(queries, 1024, [&](int64_t first, unsigned n) {
      if (cuts) hipLaunchKernelGGL((k_draw_small<TYPE, true>), dim3(n), dim3(1024), 0, st, a, first);
      else hipLaunchKernelGGL((k_draw_small<TYPE, false>), dim3(n), dim3(1024), 0, st, a, first);
    });
    return;
  }
  const bool greedy = !a.temperatures && a.temperature == 0.f;
  const bool all = a.top_ks || (!greedy && (a.top_k == 0 || a.top_k >= a.rows)), cuts = a.top_ps || a.top_p < 1.f;
  sm_launches(queries * a.chunks, 256, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_scan<TYPE>, dim3(n), dim3(256), 0, st, a, first); });
  if (all) {
    if (cuts) {
      sm_launches(queries * a.chunks, 256, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_hist<TYPE>, dim3(n), dim3(256), 0, st, a, first); });
      sm_launches(queries, 1024, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_range, dim3(n), dim3(1024), 0, st, a, first); });
    }
    sm_launches(queries * a.chunks, 256, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_weigh<TYPE>, dim3(n), dim3(256), 0, st, a, first); });
  }
  sm_launches(queries, 1024, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_rows<TYPE>, dim3(n), dim3(1024), 0, st, a, first); });
  sm_launches(queries, 1024, [&](int64_t first, unsigned n) { hipLaunchKernelGGL(k_draw_slowly<TYPE>, dim3(n), dim3(1024), 0, st, a, first); });
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
  a.chunks = L.chunks; a.chunk_rows = L.chunk_rows; a.blocks = L.blocks; a.merge = L.merge; a.groups = L.groups; a.list = L.list;
  char* const ws = (char*)workspace;
  a.stats = (DrawChunk*)(ws + L.stats); a.maxima = (unsigned*)(ws + L.maxima); a.hist = (unsigned*)(ws + L.hist); a.hist_bits = L.hist_bits; a.range = (DrawRange*)(ws + L.range);
  a.totals = (draw_u64*)(ws + L.totals); a.kept = (unsigned*)(ws + L.kept); a.listed = (unsigned*)(ws + L.listed); a.undone = (unsigned*)(ws + L.undone); a.lists = (draw_u64*)(ws + L.lists);
  a.mass = (draw_u64*)(ws + L.mass); a.mass_pitch = L.mass_pitch;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (p->dtype == MAR_DTYPE_FP32) launch_draws<0>(a, p->num_queries, st);
  else if (p->dtype == MAR_DTYPE_BF16) launch_draws<1>(a, p->num_queries, st);
  else launch_draws<2>(a, p->num_queries, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("sampling kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
