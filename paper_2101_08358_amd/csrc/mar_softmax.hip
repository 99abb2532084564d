// Log probabilities over all rows of a table: of given answers, with the distribution's entropy and its most probable rows (gfx950).
//
// Pass 0 (mar_softmax_dev.h) leaves statistics per query and part of the table, and of every group of 16 group_tiles rows the largest
// score, with the register it came from, and the second largest.  k_answer joins the parts, a workgroup per query.  The most
// probable rows lie in the groups with the largest maxima.  The rows behind the maxima are scored in 64 bits; only where a
// group's second largest score reaches the k-th best of those are its other rows looked at too, and only where the least maximum of
// the groups taken reaches it are there more groups to look at.  (All rows of the best groups scored again, 16 each: 4,096 queries,
// 131,072 rows of 400 columns, 16 best rows 367 us, for 1 GB of rows read at random.)
#include "mar_softmax_dev.h"

// Queries above which the matrices are laid out as images first, us rows / images: fp32, 120,000 rows of 100 columns, 128 queries 54 /
// 62, 256: 74 / 77, 384: 98 / 92; 1,000,000 rows 244 / 416, 400 / 473, 574 / 592; 100,000 rows of 400 columns 125 / 143, 190 / 179,
// 229 / 209.  bf16, 256, 384 and 512 queries: 46 / 51, 60 / 62, 69 / 70; 191 / 246, 255 / 301, 341 / 368; 71 / 83, 96 / 102, 113 / 115.
constexpr int sm_rows_most(int type) { return type == MAR_DTYPE_FP32 ? 256 : 512; }
#define SM_MARGIN 12              // groups, and rows, kept beyond the number asked for: few scores that fp32 less four bits cannot tell apart

struct AnswerArgs {
  const void *Q, *W; int64_t q_stride, w_stride, rows;
  int32_t n, dim, parts, num_top, group_tiles;
  int64_t ngroups, half;           // groups a half, and as many places as a half's have in a query's row
  float scale; double unscale;
  const int32_t* targets;
  const uint32_t* allowed; int64_t allowed_stride;
  const float4* stats; const float *first, *second;
  float c;                         // scale log2(e)
  float *log_probs, *entropy, *top_log_probs; int32_t* top_ids;
};

// Ascending with the value: -inf, NaN: 0, never chosen.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v);
  if (!(v > -__builtin_inff())) return 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

#define SM_CAP 96                 // candidates that are ranked by comparing all with all

// The best `want` entries seen so far, in order: by descending key, then ascending id.
struct TopList {
  __attribute__((aligned(16))) unsigned long long cand[SM_CAP + MAR_MAX_TOP + SM_MARGIN + 8], best[MAR_MAX_TOP + SM_MARGIN];   // key << 32 | ~id
  uint32_t group[64], threshold;
  int cnt[2][16], num, have;
};

// Adds the entries of a chunk to the list: R a thread (n in all, thread tid holds entries tid, NT + tid, ..), key[j] (0: none) with
// id(j).  The threshold is the want-th largest of the maxima of 64 groups of threads, which at least `want` entries reach and
// rarely more than SM_CAP.  Else one that between `want` and SM_CAP reach is found by bisection; where equal keys straddle it, a
// second bisection over their ids takes the lowest.  All threads of the workgroup.
template <int NT, int R, typename F>
__device__ __forceinline__ void add_entries(TopList& top, const uint32_t (&key)[R], F id, int n, int want) {
  constexpr int NW = NT / 64, PER = NT / 64;               // threads to a group
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  uint32_t mine = 0u;
#pragma unroll
  for (int j = 0; j < R; ++j) if (R == 1 || j * NT < n) mine = max(mine, key[j]);
#pragma unroll
  for (int o = 1; o < PER; o <<= 1) mine = max(mine, (uint32_t)__shfl_xor((int)mine, o));
  __syncthreads();
  if (tid % PER == 0) top.group[tid / PER] = mine;
  if (tid == 0) top.num = 0;
  __syncthreads();
  // a full list's last entry bounds what can still enter
  const int old = top.have;
  const uint32_t floor_key = old == want ? max((uint32_t)(top.best[want - 1] >> 32), 1u) : 1u;
  if (old < want && wave == 0) {
    const uint32_t v = top.group[lane];
    int rank = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) {
      const uint32_t w = (uint32_t)__builtin_amdgcn_readlane((int)v, j);
      rank += w > v || (w == v && j < lane) ? 1 : 0;
    }
    if (rank == want - 1) top.threshold = v;
  }
  __syncthreads();
  uint32_t x = old == want ? floor_key : max(top.threshold, 1u);
  uint32_t tie = 0u, id_end = ~0u;                         // of the entries with key `tie` those with an id below id_end
  auto collect = [&]() {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (R == 1 || j * NT < n) {
        if (key[j] >= x || (tie && key[j] == tie && id(j) < id_end)) {
          const int at = atomicAdd(&top.num, 1);
          if (at < SM_CAP) top.cand[at] = (unsigned long long)key[j] << 32 | (uint32_t)~id(j);
        }
      }
    }
    __syncthreads();
  };
  collect();
  if (top.num > SM_CAP) {                                  // uniform
    int turn = 0;
    auto total = [&](int c) {                              // c: of the wave
      if (lane == 0) top.cnt[turn & 1][wave] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) c += top.cnt[turn & 1][w];
      ++turn;
      return c;
    };
    auto count = [&](uint32_t y) {
      int c = 0;
#pragma unroll
      for (int j = 0; j < R; ++j) if (R == 1 || j * NT < n) c += __popcll(__builtin_amdgcn_ballot_w64(key[j] >= y));
      return total(c);
    };
    uint32_t lo = x, hi = ~0u;                             // more than SM_CAP reach lo, fewer than `want` hi
    while (hi - lo > 1u) {
      x = lo + (hi - lo) / 2;
      const int c = count(x);
      if (c > SM_CAP) lo = x; else if (c < want) hi = x; else break;
    }
    if (hi - lo <= 1u) {
      x = hi; tie = lo;
      const int above = count(x);
      uint32_t a = 0u, b = ~0u;                            // ids below a: too few, below b: too many
      while (true) {
        id_end = a + (b - a) / 2;
        int c = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) if (R == 1 || j * NT < n) c += __popcll(__builtin_amdgcn_ballot_w64(key[j] == tie && id(j) < id_end));
        c = above + total(c);
        if (c < want) a = id_end; else if (c > SM_CAP) b = id_end; else break;
      }
    }
    __syncthreads();
    if (tid == 0) top.num = 0;
    __syncthreads();
    collect();
  }
  const int fresh = min(top.num, SM_CAP), all = fresh + old;
  static_assert(MAR_MAX_TOP + SM_MARGIN + 8 <= 64 && NT >= 64, "a thread for every entry of the list");
  if (tid < old) top.cand[fresh + tid] = top.best[tid];
  if (tid >= old && tid < old + 8) top.cand[fresh + tid] = 0ull;
  __syncthreads();
  for (int e = tid; e < (all + 63) / 64 * 64; e += NT) {   // whole waves; there may be more entries than threads
    const unsigned long long k = e < all ? top.cand[e] : ~0ull;
    int rank = 0;
    for (int j0 = 0; j0 < all; j0 += 8) {                  // eight reads in flight; entries from `all` on are 0
      unsigned long long w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = top.cand[j0 + j];
#pragma unroll
      for (int j = 0; j < 8; ++j) rank += w[j] > k ? 1 : 0;
    }
    if (e < all && rank < want) top.best[rank] = k;
  }
  if (tid == 0) top.have = min(all, want);
  __syncthreads();
}

__device__ __forceinline__ double at_least_0(double v) { return v < 0.0 ? 0.0 : v; }        // NaN stays
// R: keys of group maxima a thread looks at together.
template <int TYPE, int NT, int R>
__global__ void __launch_bounds__(NT)
k_answer(AnswerArgs a) {
  typedef typename RowType<TYPE>::T T;
  constexpr int MAXW = MAR_MAX_TOP + SM_MARGIN, NW = NT / 64, BATCH = NT / 8 < 64 ? 64 : NT / 8, SL = NT / BATCH, EPT = (BATCH + MAXW + BATCH - 1) / BATCH;
  constexpr int QN = (MAR_MAX_DIM + 7) / 8 * 8;
  __shared__ float s_m[NW], s_l[NW], s_a[NW];
  __shared__ __attribute__((aligned(16))) float qs[QN];
  __shared__ TopList top;
  __shared__ double exact[BATCH + MAXW], qn, s_lse;        // kept where registers are few
  __shared__ unsigned long long reach;
  __shared__ uint32_t exact_row[BATCH + MAXW];
  constexpr int LIST = NT > MAXW ? NT : MAXW;
  __shared__ int groups[LIST], again[LIST], num_exact;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t q = blockIdx.x;
  const T* qr = (const T*)a.Q + q * a.q_stride;
  const T* W = (const T*)a.W;
  const uint32_t* allowed = a.allowed ? a.allowed + q * a.allowed_stride : nullptr;
  auto is_allowed = [&](int64_t row) { return !allowed || (allowed[row >> 5] >> (row & 31) & 1u); };
  // group maxima of a chunk: element e of the query's row [2][half] belongs to group 2 (e % half) + e / half
  const float* gm = a.first + q * 2 * a.half;
  auto load_keys = [&](int64_t g0, uint32_t (&key)[R]) {
    float v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t e = g0 + j * NT + tid;
      v[j] = e < 2 * a.half && (e < a.half ? e : e - a.half) < a.ngroups ? gm[e] : -__builtin_inff();
    }
#pragma unroll
    for (int j = 0; j < R; ++j) key[j] = v[j] > 0.99f * SM_NO_REF ? order_key(v[j]) & ~15u : 0u;
  };
  uint32_t key[R];
  if (a.num_top) load_keys(0, key);

  // ---- statistics of all parts
  float m = SM_NO_REF, l = 0.f, s = 0.f;
  for (int p = tid; p < a.parts; p += NT) { const float4 v = a.stats[(size_t)p * a.n + q]; sm_join(m, l, s, v.x, v.y, v.z); }
  if (a.parts > 1) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sm_join(m, l, s, __shfl_xor(m, o), __shfl_xor(l, o), __shfl_xor(s, o));
  }
  if (lane == 0) { s_m[wave] = m; s_l[wave] = l; s_a[wave] = s; }
  for (int c = tid; c < QN; c += NT) qs[c] = c < a.dim ? (float)qr[c] : 0.f;
  if (tid == 0) top.have = 0;
  __syncthreads();
  m = s_m[0]; l = s_l[0]; s = s_a[0];
  for (int w = 1; w < NW && w * 64 < a.parts; ++w) sm_join(m, l, s, s_m[w], s_l[w], s_a[w]);
  const double lse = (double)m * a.unscale + log_of_sum(l);

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
      s_lse = lse;
      if (a.log_probs) a.log_probs[q] = !has ? 0.f : (is_allowed(t) ? (float)at_most_0(dot * (double)a.scale - lse) : -__builtin_inff());
      if (a.entropy) a.entropy[q] = l == 0.f ? 0.f : (float)at_least_0(log_of_sum(l) - 0.69314718055994530942 * ((double)s / (double)l));
    }
  }
  if (a.num_top == 0) return;

  // ---- groups with the largest maxima; among equal ones the first
  const int want = a.num_top + SM_MARGIN;
  for (int64_t g0 = 0;;) {
    add_entries<NT, R>(top, key, [&](int j) {
      const int64_t e = g0 + j * NT + tid;
      return (uint32_t)(e < a.half ? 2 * e : 2 * (e - a.half) + 1);
    }, (int)min((int64_t)NT * R, 2 * a.half - g0), want);
    g0 += (int64_t)NT * R;
    if (g0 >= 2 * a.half) break;
    load_keys(g0, key);
  }
  // ---- the rows behind their maxima in 64 bits (with more than one tile to a group, that register's row of every tile)
  const int ngr = top.have, G = a.group_tiles;
  if (tid < ngr) groups[tid] = (int)~(uint32_t)top.best[tid];
  if (tid == 0) { num_exact = 0; reach = 0ull; }
  __syncthreads();
  auto element = [&](int grp) { return (int64_t)(grp & 1) * a.half + (grp >> 1); };
  auto row_of = [&](int grp, int tile, int r) { return ((int64_t)(grp >> 1) * G + tile) * SM_TY + 8 * (r >> 2) + 4 * (grp & 1) + (r & 3); };
  constexpr int UL = NT <= 256 ? 4 : (TYPE == MAR_DTYPE_FP32 ? 2 : 3);   // as registers allow
  // Scores items [0, n): row(item) or -1, eight lanes an item.  The list is put in order and cut back to its best `want` after every
  // BATCH items of which some come before its num_top-th.
  int listed = 0;                                          // entries in order
  auto score_items = [&](int n, auto row) {
    for (int b0 = 0; b0 < n; b0 += BATCH) {
      for (int e0 = b0; e0 < min(n, b0 + BATCH); e0 += NT / 8) {
        const int e = e0 + (tid >> 3);
        int64_t rw = e < n ? row(e) : -1;
        if (rw >= a.rows || (rw >= 0 && !is_allowed(rw))) rw = -1;
        double dot = 0.0, n2 = 0.0;
        if (rw >= 0) {
          const T* wr = W + rw * a.w_stride;
          for (int u0 = 0; 64 * u0 < a.dim; u0 += UL) {    // uniform; UL loads in flight
            float v[UL][8];
#pragma unroll
            for (int u = 0; u < UL; ++u) load8<TYPE>(wr, 8 * (8 * (u0 + u) + (tid & 7)), a.dim, v[u]);
#pragma unroll
            for (int u = 0; u < UL; ++u) {
              const int c = min(8 * (8 * (u0 + u) + (tid & 7)), QN - 8);     // values from dim on are zeros
              const float4 qa = *reinterpret_cast<const float4*>(qs + c), qb = *reinterpret_cast<const float4*>(qs + c + 4);
              const float qv[8] = {qa.x, qa.y, qa.z, qa.w, qb.x, qb.y, qb.z, qb.w};
#pragma unroll
              for (int j = 0; j < 8; ++j) { dot = __builtin_fma((double)qv[j], (double)v[u][j], dot); n2 = __builtin_fma((double)v[u][j], (double)v[u][j], n2); }
            }
          }
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) { dot += __shfl_xor(dot, o); n2 += __shfl_xor(n2, o); }
        const int end = a.num_top - 1;
        if ((tid & 7) == 0 && rw >= 0 && dot == dot) {
          atomicMax(&reach, (unsigned long long)__double_as_longlong(n2));   // the largest squared norm (fp32 squares may leave the floats' range)
          if (listed <= end || dot > exact[end] || (dot == exact[end] && rw < exact_row[end])) {
            const int at = atomicAdd(&num_exact, 1);       // below BATCH + MAXW
            exact[at] = dot; exact_row[at] = (uint32_t)rw;
          }
        }
      }
      __syncthreads();
      const int have = num_exact;
      if (have == listed) { __syncthreads(); continue; }   // uniform; all have read the number
      // an entry's rank: SL threads each compare it with a part of the others
      double v[EPT];
      uint32_t rw[EPT];
      int rank[EPT];
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const int e = i * BATCH + tid / SL;
        rank[i] = want;
        if (i * BATCH < have) {                            // uniform
          v[i] = exact[min(e, have - 1)]; rw[i] = exact_row[min(e, have - 1)]; rank[i] = 0;
#pragma unroll 4
          for (int j = tid % SL; j < have; j += SL) rank[i] += exact[j] > v[i] || (exact[j] == v[i] && exact_row[j] < rw[i]) ? 1 : 0;
#pragma unroll
          for (int o = 1; o < SL; o <<= 1) rank[i] += __shfl_xor(rank[i], o);
          if (e >= have) rank[i] = want;
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < EPT; ++i) if (rank[i] < want && tid % SL == 0) { exact[rank[i]] = v[i]; exact_row[rank[i]] = rw[i]; }
      listed = __builtin_amdgcn_readfirstlane(min(have, want));
      if (tid == 0) num_exact = listed;
      __syncthreads();
    }
  };
  // What a pass's score is off at most: MFMA chains of up to 75 products in fp32 and pairs of f16, 2^-15 of |q| |row| (2^-20 as measured; so
  // the rows' lengths need not be known beyond those that are scored), and the four bits that hold the register's number.
  if (wave == 0) {
    double n2 = 0.0;
    for (int c = lane; c < a.dim; c += 64) n2 = __builtin_fma((double)qs[c], (double)qs[c], n2);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) n2 += __shfl_xor(n2, o);
    if (lane == 0) qn = n2;                                // read behind a barrier of score_items
  }
  // The k-th best score so far less that, in the passes' log2 units; -inf while there are fewer.
  auto bar = [&]() {
    if (num_exact < a.num_top) return -__builtin_inff();
    const double kth = exact[a.num_top - 1] * (double)a.c;
    return (float)(kth - (fabs(kth) * 0x1p-16 + sqrt(qn) * sqrt(__longlong_as_double((long long)reach)) * (double)a.c * 0x1p-15));
  };
  // Groups of the list first, then (rare: many scores that the passes cannot tell apart) all others whose maxima reach the bar, a chunk
  // of NT groups at a time.
  const int all = (int)(2 * a.half);
  int n = ngr, e0 = 0;
  while (true) {
    if (n) {                                               // uniform
      score_items(n * G, [&](int e) {
        const int grp = groups[e / G];
        return row_of(grp, e % G, (int)(__float_as_uint(gm[element(grp)]) & 15u));
      });
      // ---- groups whose second largest score may reach the k-th best
      const float least = bar();
      if (tid == 0) top.num = 0;
      __syncthreads();
      if (tid < n) {
        const float two = a.second[q * 2 * a.half + element(groups[tid])] * a.c;
        if (two > 0.99f * SM_NO_REF * a.c && two >= least) again[atomicAdd(&top.num, 1)] = groups[tid];
      }
      __syncthreads();
      score_items(top.num * G * 16, [&](int e) {
        const int grp = again[e / (G * 16)], r = e & 15, one = (int)(__float_as_uint(gm[element(grp)]) & 15u);
        return r == one ? (int64_t)-1 : row_of(grp, (e >> 4) % G, r);
      });
    }
    if (top.have < want || e0 >= all) break;               // every group was in the list, or has been looked at
    if (qn == 0.0 || reach == 0ull) break;                 // all scores are zeros, as measured: the list has the lowest ids
    const float least = bar();
    const unsigned long long last = top.best[want - 1];    // groups up to this one have been seen, in the order of the list
    if (e0 == 0) {
      const uint32_t key = (uint32_t)(last >> 32) | 15u;   // the least maximum in the list
      if (__uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key) * a.c < least) break;
    }
    __syncthreads();
    if (tid == 0) top.num = 0;
    __syncthreads();
    const int e = e0 + tid, half = (int)a.half;
    if (e < all && (e < half ? e : e - half) < a.ngroups) {
      const float v = gm[e];
      const uint32_t key = v > 0.99f * SM_NO_REF ? order_key(v) & ~15u : 0u, id = (uint32_t)(e < half ? 2 * e : 2 * (e - half) + 1);
      if (key && ((unsigned long long)key << 32 | (uint32_t)~id) < last && v * a.c >= least) groups[atomicAdd(&top.num, 1)] = (int)id;
    }
    __syncthreads();
    n = top.num;
    e0 += NT;
  }
  const int have = min(num_exact, a.num_top);
  for (int e = tid; e < a.num_top; e += NT) {
    a.top_ids[q * a.num_top + e] = e < have ? (int32_t)exact_row[e] : -1;
    a.top_log_probs[q * a.num_top + e] = e < have ? (float)at_most_0(exact[e] * (double)a.scale - s_lse) : -__builtin_inff();
  }
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
SmPlan sm_plan(int dtype, int dim, int pass, int mode, int64_t n_x, int64_t n_y, int multiple) {
  SmPlan r;
  const int nk = sm_nk(dim);
  r.ntiles = (int32_t)((n_y + SM_TY - 1) / SM_TY);
  if (mode == SM_FEW) {                                    // every wave that the device holds, at least a tile each
    const int64_t tile = (int64_t)SM_TY * sp_pitch(nk) * (dtype == MAR_DTYPE_FP32 ? 2 : 1);
    const int64_t a_cu = 4 * sm_waves_of(dtype, nk, 0, SM_FEW), fit = 160 * 1024 / (tile + 1024), slots = 256 * (a_cu < fit ? a_cu : fit);
    int64_t tps = (r.ntiles + slots - 1) / slots;
    if (tps < 1) tps = 1;
    tps = (tps + multiple - 1) / multiple * multiple;
    r.stripes = 1; r.tps = (int32_t)tps; r.parts = (int32_t)((r.ntiles + tps - 1) / tps);
    return r;
  }
  r.stripes = (int32_t)((n_x + 127) / 128);
  const int64_t slots = 256 * sm_waves_of(dtype, nk, pass, mode);
  int64_t best = INT64_MAX;
  r.parts = 1; r.tps = r.ntiles;
  const int most = pass == 0 ? 1024 : MAR_SOFTMAX_MAX_PARTS;
  const int64_t room = (sm_most_blocks(256) - 7) / (r.stripes > 0 ? r.stripes : 1);    // one launch, its units rounded up to eights
  for (int k = 1; k <= most && k <= r.ntiles && k <= room; k += 1 + k / 32) {          // the host has some microseconds
    int64_t tps = (r.ntiles + k - 1) / k;
    tps = (tps + multiple - 1) / multiple * multiple;
    const int64_t parts = (r.ntiles + tps - 1) / tps;
    const int64_t cost = (r.stripes * parts + slots - 1) / slots * (tps + (pass == 0 ? 4 : 8));
    if (cost < best) { best = cost; r.parts = (int32_t)parts; r.tps = (int32_t)tps; }
  }
  return r;
}

// Tiles to a group: one while a query has no more than 4,096 groups, then as many as leave the rows behind the best groups' maxima to
// one round of a workgroup of 1,024 (128 rows; a round costs as much as looking through 40,000 maxima).
static int group_tiles(const mar_softmax* p, int num_top) {
  const int64_t ntiles = (p->num_rows + SM_TY - 1) / SM_TY, most = 128 / (num_top + SM_MARGIN);
  const int64_t g = (ntiles + 2047) / 2048;
  return (int)(g < most ? g : most);
}

struct ProbsLayout { size_t stats, first, second, qtiles, qexps, wtiles, wexps, bytes; SmPlan p0; int group_tiles; int64_t ngroups, half; int mode; };
static ProbsLayout probs_layout(const mar_softmax* p, int num_top) {
  ProbsLayout L;
  L.group_tiles = num_top ? group_tiles(p, num_top) : 1;
  L.mode = p->num_queries <= 32 && sm_nk(p->dim) <= 16 ? SM_FEW : (p->num_queries > sm_rows_most(p->dtype) ? SM_IMAGES : SM_ROWS);
  // group maxima are stored four groups at a time, but for few queries
  L.p0 = sm_plan(p->dtype, p->dim, 0, L.mode, p->num_queries, p->num_rows, num_top ? (L.mode == SM_FEW ? 1 : 4) * L.group_tiles : 1);
  L.ngroups = num_top ? (L.p0.ntiles + L.group_tiles - 1) / L.group_tiles : 0;
  L.half = (L.ngroups + 3) / 4 * 4 + 8;                    // queries' rows not a power of two apart
  const size_t T = (size_t)p->num_queries;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  L.stats = take((size_t)L.p0.parts * T * sizeof(float4));
  L.first = take(num_top ? T * 2 * (size_t)L.half * 4 : 0);
  L.second = take(num_top ? T * 2 * (size_t)L.half * 4 : 0);
  L.qtiles = L.qexps = L.wtiles = L.wexps = at;
  if (L.mode == SM_IMAGES) {
    L.qtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_queries)); L.qexps = take(sm_exps_bytes(p->num_queries));
    L.wtiles = take(sm_image_bytes(p->dtype, p->dim, p->num_rows)); L.wexps = take(sm_exps_bytes(p->num_rows));
  }
  L.bytes = at > 256 ? at : 256;
  return L;
}

template <int TYPE, int MODE> static void launch_nk(const SmArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.units + 7) / 8 * 8)), block(sm_threads(MODE));
  switch (sm_nk(a.dim)) {
    case 2: hipLaunchKernelGGL((k_softmax<TYPE, 2, 0, MODE>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_softmax<TYPE, 4, 0, MODE>), grid, block, 0, st, a); break;
    case 7: hipLaunchKernelGGL((k_softmax<TYPE, 7, 0, MODE>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((k_softmax<TYPE, 8, 0, MODE>), grid, block, 0, st, a); break;
    case 12: hipLaunchKernelGGL((k_softmax<TYPE, 12, 0, MODE>), grid, block, 0, st, a); break;
    case 16: hipLaunchKernelGGL((k_softmax<TYPE, 16, 0, MODE>), grid, block, 0, st, a); break;
    default: if constexpr (MODE != SM_FEW) hipLaunchKernelGGL((k_softmax<TYPE, 25, 0, MODE>), grid, block, 0, st, a); break;
  }
}
template <int TYPE> static void launch_pack(const SmPackArgs& a, const SmPackArgs& b, hipStream_t st) {
  sm_launches(sm_tiles(a.n) + sm_tiles(b.n), 256, [&](int64_t first, unsigned blocks) {
    const dim3 grid(blocks), block(256);
    const int at = (int)first;
    switch (sm_nk(a.dim)) {
      case 2: hipLaunchKernelGGL((k_softmax_pack<TYPE, 2>), grid, block, 0, st, a, b, at); break;
      case 4: hipLaunchKernelGGL((k_softmax_pack<TYPE, 4>), grid, block, 0, st, a, b, at); break;
      case 7: hipLaunchKernelGGL((k_softmax_pack<TYPE, 7>), grid, block, 0, st, a, b, at); break;
      case 8: hipLaunchKernelGGL((k_softmax_pack<TYPE, 8>), grid, block, 0, st, a, b, at); break;
      case 12: hipLaunchKernelGGL((k_softmax_pack<TYPE, 12>), grid, block, 0, st, a, b, at); break;
      case 16: hipLaunchKernelGGL((k_softmax_pack<TYPE, 16>), grid, block, 0, st, a, b, at); break;
      default: hipLaunchKernelGGL((k_softmax_pack<TYPE, 25>), grid, block, 0, st, a, b, at); break;
    }
  });
}
hipError_t sm_pack(int dtype, const SmPackArgs& a, const SmPackArgs& b, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_pack<0>(a, b, st); else if (dtype == MAR_DTYPE_BF16) launch_pack<1>(a, b, st); else launch_pack<2>(a, b, st);
  return hipGetLastError();
}
size_t sm_image_bytes(int dtype, int dim, int64_t rows) {
  const int nk = sm_nk(dim);
  return (size_t)((rows + SM_TY - 1) / SM_TY) * SM_TY * sp_pitch(nk) * (dtype == MAR_DTYPE_FP32 ? 2 : 1);
}
template <int MODE> static hipError_t launch_stats(int dtype, const SmArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_nk<0, MODE>(a, st); else if (dtype == MAR_DTYPE_BF16) launch_nk<1, MODE>(a, st); else launch_nk<2, MODE>(a, st);
  return hipGetLastError();
}

// Threads per query: all that hide a query's own latency where there are few, and as many as leave all queries resident at once
// (twelve waves a CU).  us a call, 64 / 128 / 256 / 1,024 threads: bf16, 120,000 rows of 100 columns, 128 queries 74 / 54 / 42 / 38,
// 512: 99 / 81 / 71 / 79, 1,000: 130 / 111 / 116 / 134, 4,000: 330 / 324 / 346 / 454; 15,000 rows, 700 queries 48 / 41 / 38 / 60, 1,000:
// 53 / 44 / 54 / 79, 2,000: 62 / 68 / 76 / 137, 4,000: 109 / 111 / 140 / 265.
template <int TYPE> static void launch_answer(const AnswerArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.n);
  if (a.n > 1536) hipLaunchKernelGGL((k_answer<TYPE, 64, 32>), grid, dim3(64), 0, st, a);
  else if (a.n > 768) hipLaunchKernelGGL((k_answer<TYPE, 128, 16>), grid, dim3(128), 0, st, a);
  else if (a.n > 256) hipLaunchKernelGGL((k_answer<TYPE, 256, 16>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_answer<TYPE, 1024, 16>), grid, dim3(1024), 0, st, a);
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
  a.first = num_top ? (float*)((char*)workspace + L.first) : nullptr;
  a.second = num_top ? (float*)((char*)workspace + L.second) : nullptr;
  a.half = L.half; a.group_tiles = L.group_tiles;
  a.allowed = allowed; a.allowed_stride = allowed_stride;
  hipError_t e;
  if (L.mode == SM_IMAGES) {
    a.ximg = sm_image((char*)workspace + L.qtiles, (char*)workspace + L.qexps, p->num_queries);
    a.yimg = sm_image((char*)workspace + L.wtiles, (char*)workspace + L.wexps, p->num_rows);
    SmPackArgs w = {}, k = {};
    w.dim = k.dim = p->dim; w.apart = k.apart = 1;
    w.src = table; w.stride = p->row_stride; w.n = (int32_t)p->num_rows; w.to = a.yimg;
    k.src = queries; k.stride = p->query_stride; k.n = p->num_queries; k.to = a.ximg;
    e = sm_pack(p->dtype, w, k, st);
    if (e != hipSuccess) { mar_set_error("image kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
    e = launch_stats<SM_IMAGES>(p->dtype, a, st);
  } else {
    e = L.mode == SM_FEW ? launch_stats<SM_FEW>(p->dtype, a, st) : launch_stats<SM_ROWS>(p->dtype, a, st);
  }
  if (e != hipSuccess) { mar_set_error("softmax kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  AnswerArgs r = {};
  r.Q = queries; r.W = table; r.q_stride = p->query_stride; r.w_stride = p->row_stride; r.rows = p->num_rows;
  r.n = p->num_queries; r.dim = p->dim; r.parts = L.p0.parts; r.num_top = num_top; r.group_tiles = L.group_tiles; r.ngroups = L.ngroups; r.half = L.half;
  r.scale = p->scale; r.unscale = (double)p->scale / (double)a.c;
  r.targets = targets; r.allowed = allowed; r.allowed_stride = allowed_stride; r.stats = a.stats; r.first = a.first; r.second = a.second; r.c = a.c;
  r.log_probs = log_probs; r.entropy = entropy; r.top_ids = top_ids; r.top_log_probs = top_log_probs;
  if (p->dtype == MAR_DTYPE_FP32) launch_answer<0>(r, st); else if (p->dtype == MAR_DTYPE_BF16) launch_answer<1>(r, st); else launch_answer<2>(r, st);
  e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("answer kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
