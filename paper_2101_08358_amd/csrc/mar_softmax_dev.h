// The contraction of mar_softmax.h on the device.
#pragma once
#include <type_traits>

#include "mar_rows_dev.h"
#include "mar_softmax.h"
#include "mar_split_dev.h"

// f(0), .., f(N - 1), unrolled whatever the body's size: the loops index registers.
template <int N, typename F> __device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (N > 0) { unrolled<N - 1>(f); f(std::integral_constant<int, N - 1>{}); }
}
// Waves per SIMD (= workgroups per CU), as registers allow.  A wave takes 32 stationary rows; 64, which halves what is read of LDS,
// left pass 0 fewer waves to hide a tile's latency (bf16, 15,000 rows of 100 columns, 256 queries 35 us, now 28; 100,000 rows of
// 256 columns, 1,000 queries 184 and 161).
constexpr int sm_waves(int type, int nk, int pass) {
  return type == MAR_DTYPE_FP32 ? (pass == 0 ? (nk <= 8 ? 3 : (nk <= 16 ? 2 : 1)) : (nk <= 4 && pass == 1 ? 3 : (nk <= 8 ? 2 : 1)))
                                : (pass == 0 ? (nk <= 8 ? 4 : (nk <= 12 ? 3 : 2)) : (nk <= 4 ? 3 : (nk <= 12 ? 2 : 1)));
}

template <int TYPE> __device__ __forceinline__ v16f sm_mfma(v8s a, v8s b, v16f c) {
  if (TYPE == MAR_DTYPE_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  return mfma32h(a, b, c);
}
// Largest finite magnitude's bits.
__device__ __forceinline__ int finite_bits(float v) { const int b = __float_as_int(v) & 0x7fffffff; return b < 0x7f800000 ? b : 0; }
// Exponent of a row or of a block of eight whose largest finite magnitude has these bits: 2^e max lies in [2^14, 2^15).  Zeros take 80:
// the second product's weights are 2^(t - e), and one far from the others' exponents would leave the floats' range.
__device__ __forceinline__ int sm_exponent(int max_bits) { return max_bits == 0 ? 80 : min(141 - (max_bits >> 23), 116); }
__device__ __forceinline__ void sm_parts8(const float (&v)[8], float scale, v8s& hi, v8s& lo) {
  v8h h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) { _Float16 a, b; sp_parts(v[e] * scale, a, b); h[e] = a; l[e] = b; }
  hi = __builtin_bit_cast(v8s, h); lo = __builtin_bit_cast(v8s, l);
}
// Largest value of eight neighbouring lanes (a staged row's), none negative, in all of them.
template <int CTRL> __device__ __forceinline__ float sm_turned(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_largest(float v) {
  v = fmaxf(v, sm_turned<0xB1>(v));                        // lane ^ 1, lane ^ 2 of four, then the eight mirrored
  v = fmaxf(v, sm_turned<0x4E>(v));
  return fmaxf(v, sm_turned<0x141>(v));
}
// Largest of a wave's eight rows' values, each the same in its eight lanes.
__device__ __forceinline__ float rows_largest(float v) {
  v = fmaxf(v, sm_turned<0x128>(v));                       // the other row of 16 lanes
  auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return fmaxf(fmaxf(lane(0), lane(16)), fmaxf(lane(32), lane(48)));
}
template <int TYPE> __device__ __forceinline__ v8s sm_round8(const float (&v)[8]) {
  if (TYPE == MAR_DTYPE_BF16) { v8b b; 
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
    return __builtin_bit_cast(v8s, b); }
  v8h h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (_Float16)v[e];
  return __builtin_bit_cast(v8s, h);
}
template <int TYPE> __device__ __forceinline__ float sm_rounded(float v) { return TYPE == MAR_DTYPE_BF16 ? (float)(__bf16)v : (float)(_Float16)v; }
__device__ __forceinline__ float pick(unsigned mask, float a, float b) {   // a where mask is all ones, b where it is 0
  return __uint_as_float((__float_as_uint(a) & mask) | (__float_as_uint(b) & ~mask));
}

template <int TYPE, int NK> struct SmGeom {
  static constexpr int PLANES = TYPE == MAR_DTYPE_FP32 ? 2 : 1;
  static constexpr int UNITS = sp_units(NK);
  static constexpr int PA = sp_pitch(NK);
  static constexpr int PLANE = SM_TY * PA;
  static constexpr int TILE = PLANES * PLANE;
  static constexpr int NP = (2 * NK + 7) / 8;              // 16-byte units a thread copies of a tile: eight threads to a row
};

// A tile on its way from memory to LDS: wave w takes rows 8 w .. 8 w + 7, eight threads to a row, a piece of 8 columns each at a time.
// fp32: the exponent of a wave's eight rows is known once all pieces are there.
template <int TYPE, int NK> struct SmStage {
  typedef SmGeom<TYPE, NK> G;
  typedef typename RowType<TYPE>::T T;
  static constexpr bool PAIRS = TYPE == MAR_DTYPE_FP32;
  row_u4 r[G::NP][G::PLANES];
  bool zero;                                               // the row is taken as zeros whatever it holds
  bool apart;                                              // it has an exponent of its own, and the eight rows' does without it
  const T* row;
  __device__ __forceinline__ void begin(const T* __restrict__ Y, int64_t stride, int n_y, int y0, int tid) {
    row = Y + (int64_t)min(y0 + (tid >> 3), n_y - 1) * stride;               // rows beyond the last are the last again
    zero = apart = false;
  }
  __device__ __forceinline__ void fetch(int p, int dim, int tid, row_u4 (&v)[G::PLANES]) const {
    const int u = (tid & 7) + 8 * p;
    if constexpr (PAIRS) {
      v[0] = take4_floats(row, 8 * u, dim);
      v[1] = take4_floats(row, 8 * u + 4, dim);
    } else {
      v[0] = take8_bits(row, 8 * u, dim);
    }
  }
  __device__ __forceinline__ void load(int p, int dim, int tid) { fetch(p, dim, tid, r[p]); }
  // FINITE: no value is infinite (a NaN makes its row's scores NaN either way)
  template <bool FINITE> __device__ __forceinline__ void put(int p, char* tile, float scale, int dim, int tid) const {
    const int u = (tid & 7) + 8 * p, y = tid >> 3;
    char* const to = tile + y * G::PA + ((16 * u) ^ (16 * sp_swizzle(G::UNITS, y)));
    if (u >= 2 * NK) return;
    if constexpr (PAIRS) {
      const row_u4 q[2] = {place4_floats(r[p][0], 8 * u, dim), place4_floats(r[p][1], 8 * u + 4, dim)};
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = zero ? 0.f : __uint_as_float(q[j >> 2][j & 3]);
      v8s hi, lo;
      if (FINITE) {
        float neg1 = -1.f;
        asm volatile("" : "+v"(neg1));
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= scale;
        split8<true>(f, neg1, hi, lo);
      } else {
        sm_parts8(f, scale, hi, lo);
      }
      *reinterpret_cast<v8s*>(to) = hi;
      *reinterpret_cast<v8s*>(to + G::PLANE) = lo;
    } else {
      *reinterpret_cast<row_u4*>(to) = zero ? (row_u4)(0u) : place8_bits(r[p][0], 8 * u, dim);
    }
  }
  // fp32: row_exps: every row's exponent; exps: of the tile's four blocks of eight rows.  OWN: all rows lie apart, exps is not written.
  template <bool OWN> __device__ __forceinline__ void store(char* tile, int* exps, int* row_exps, int dim, int tid) {
    float scale = 1.f;
    if constexpr (PAIRS) {
      // columns that a piece at the row's end holds besides its own belong to the same row: they may be measured too
      float big = 0.f;
#pragma unroll
      for (int p = 0; p < G::NP; ++p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(__uint_as_float(r[p][j >> 2][j & 3])));
      }
      if (zero) big = 0.f;
      const bool finite = !__any(__float_as_int(big) >= 0x7f800000);       // uniform
      if (!finite) {                                       // an infinity: the exponent of what is finite
        int most = 0;
#pragma unroll
        for (int p = 0; p < G::NP; ++p) {
#pragma unroll
          for (int j = 0; j < 8; ++j) most = max(most, finite_bits(__uint_as_float(r[p][j >> 2][j & 3])));
        }
        big = __int_as_float(zero ? 0 : most);
      }
      big = row_largest(big);
      int e = sm_exponent(__float_as_int(big));
      if (!OWN) {
        const int block = sm_exponent(__float_as_int(rows_largest(apart ? 0.f : big)));
        if ((tid & 63) == 0) exps[tid >> 6] = block;
        e = apart ? e : block;
      }
      if ((tid & 7) == 0) row_exps[tid >> 3] = e;
      scale = __builtin_ldexpf(1.f, e);
      if (!finite) {
#pragma unroll
        for (int p = 0; p < G::NP; ++p) put<false>(p, tile, scale, dim, tid);
        return;
      }
    }
#pragma unroll
    for (int p = 0; p < G::NP; ++p) put<true>(p, tile, scale, dim, tid);
  }
};

// Joins two parts' statistics: reference, sum of weights, sum of weights times (t - reference).
__device__ __forceinline__ void sm_join(float& m, float& l, float& s, float m2, float l2, float s2) {
  const float to = fmaxf(m, m2), d1 = m - to, d2 = m2 - to, f1 = __builtin_amdgcn_exp2f(d1), f2 = __builtin_amdgcn_exp2f(d2);
  const float sa = l != 0.f ? f1 * __builtin_fmaf(d1, l, s) : 0.f, sb = l2 != 0.f ? f2 * __builtin_fmaf(d2, l2, s2) : 0.f;
  l = l * f1 + l2 * f2; s = sa + sb; m = to;
}
// Floats as integers of the same order.
#define SM_NO_OWN INT32_MIN
__device__ __forceinline__ int own_key(float v) { const int b = __float_as_int(v); return b < 0 ? b ^ 0x7fffffff : b; }
__device__ __forceinline__ float own_float(int k) { return __int_as_float(k < 0 ? k ^ 0x7fffffff : k); }
// Softmax weights in fp16 (and as pairs of f16) lie between 2^-24 and 2^16: the reference is put 12 below the largest exponent met
// and moves when one exceeds it by more than 15; what is 2^-36 of the largest weight is lost to the second product (never to the sum).
// References are integers: moving one, and joining parts, multiplies by powers of two only, and a weight of 1 stays exact.  In pass 0,
// without a second product, a lane's reference is its largest score: the entropy of a confident query is what the other rows' weights
// add to log 1, and to 0 (with references 12 below, differences of numbers near 12 log 2: off by 5e-7).
#define SM_ABOVE 15.f
#define SM_BELOW 12.f
#define SM_SUM_ABOVE 90.f         // 2^29 rows' sum stays a float; a block of zeros (exponent 80) beside rows of up to 2^20 moves nothing
#define SM_CHAIN 16               // tiles whose weights are summed before their sum is added to the part's: chains of fp32 sums stay short

// How the streamed rows come: SM_IMAGES: both matrices as images.  SM_ROWS: from the rows themselves, a tile staged by the
// workgroup (a table that few stripes of queries meet is not worth laying out).  SM_FEW: the queries fit one wave's registers;
// every wave is a workgroup of its own and streams tiles of its own, without a barrier, at the rate of the memory.
#define SM_ROWS 0
#define SM_IMAGES 1
#define SM_FEW 2
constexpr int sm_threads(int mode) { return mode == SM_FEW ? 64 : 256; }
// Waves per SIMD by mode: staging takes registers of its own.
constexpr int sm_waves_of(int type, int nk, int pass, int mode) {
  const bool wide = type == MAR_DTYPE_FP32;
  return mode == SM_IMAGES ? sm_waves(type, nk, pass)
         : mode == SM_FEW  ? (wide ? (nk <= 4 ? 2 : 1) : (nk <= 8 ? 3 : (nk <= 12 ? 2 : 1)))
                           : (wide ? (nk <= 4 ? 3 : (nk <= 12 ? 2 : 1)) : (nk <= 8 ? 4 : 2));
}
template <int TYPE, int NK, int PASS, int MODE>
__global__ void __launch_bounds__(sm_threads(MODE)) __attribute__((amdgpu_waves_per_eu(sm_waves_of(TYPE, NK, PASS, MODE), sm_waves_of(TYPE, NK, PASS, MODE))))
k_softmax(SmArgs a) {
  typedef SmGeom<TYPE, NK> G;
  typedef typename RowType<TYPE>::T T;
  constexpr bool PAIRS = TYPE == MAR_DTYPE_FP32;
  constexpr bool IMG = MODE == SM_IMAGES, FEW = MODE == SM_FEW;
  constexpr bool SECOND = PASS != 0;
  constexpr int NO = SECOND ? (NK + 1) / 2 : 1;            // 32-column blocks of the output
  constexpr bool REFS = PASS != 2 || TYPE != MAR_DTYPE_BF16 || NK > 16;   // weights relative to a reference (bf16 does without; the widest rows' registers do not)
  constexpr int PL = G::PLANES;
  static_assert(IMG || PASS == 0, "passes with a second product take images");
  constexpr int NB = FEW ? 1 : 2;                          // tiles in LDS
  __shared__ __attribute__((aligned(1024))) char smem[NB * G::TILE];
  // fp32: exponents of a tile's rows; of its four blocks of eight, which a second product over the rows needs to share
  constexpr int NE = PASS == 0 ? SM_TY : 4;
  __shared__ __attribute__((aligned(16))) int exps[2][NE];
  // pass 2, per query of a tile: f = log2(|u| / sum of its weights), m its reference (16-bit types: f - m and nothing)
  __shared__ __attribute__((aligned(16))) float rows_m[2][SM_TY], rows_f[2][SM_TY], rows_u[2][SM_TY];
  __shared__ __attribute__((aligned(16))) int rows_t[2][SM_TY];
  __shared__ unsigned rows_neg[2], rows_none[2];           // queries with a negative u; without weight (or beyond the last)
  __shared__ __attribute__((aligned(16))) short rows_keep[2][SM_TY];       // 0 for those without, else all ones
  __shared__ int own[PASS == 2 && REFS ? 128 : 1];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, m = lane & 31, g = lane >> 4, i = lane & 15;
  // workgroups of one part of the streamed rows share an XCD's L2: XCD j takes a contiguous eighth of the (part, stripe) units
  const int unit = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  if (unit >= a.units) return;
  const int part = unit / a.nstripes, stripe = unit - part * a.nstripes;
  const int ntiles_all = (int)(((int64_t)a.n_y + SM_TY - 1) / SM_TY);
  const int t_begin = part * a.tps, t_end = min(ntiles_all, t_begin + a.tps);
  const int64_t x_first = FEW ? 0 : (int64_t)stripe * 128 + wave * 32;
  const int dim = a.dim;

  // zeros: units beyond the columns that a tile's copies write
  if (!IMG) for (int k = tid * 16; k < NB * G::TILE; k += sm_threads(MODE) * 16) *reinterpret_cast<row_u4*>(smem + k) = (row_u4)(0u);
  constexpr int NSG = FEW ? 4 : 1;                         // blocks of eight rows a wave stages
  SmStage<TYPE, NK> stage[NSG];
  const T* Y = (const T*)a.Y;
  // images: copied by loads that write LDS, 1 KB a wave instruction; nothing but the end of the tile waits for them
  int token = 0;
  constexpr int NCW = (G::TILE / 1024 + 3) / 4;            // pieces a wave
  auto copy = [&](int t, int buf, int p) {
    const int piece = 4 * p + wave;
    if (piece < G::TILE / 1024)
      buf_load4_to_lds(buf_words(a.yimg.tiles + (size_t)t * G::TILE, G::TILE), lds_address_b(smem) + buf * G::TILE + piece * 1024, lane * 16, piece * 1024, token);
  };
  int ye = 0;                                              // exponent lane % NE of the tile on its way
  auto ask_exps = [&](int t) { if (IMG && PAIRS) ye = (PASS == 0 ? a.yimg.row_exps : a.yimg.exps)[NE * (int64_t)t + (lane & (NE - 1))]; };
  float q_m = 0.f, q_f = 0.f, q_u = 0.f;
  int q_t = -1;
  auto load_rows = [&](int y0) {
    if (PASS == 2 && tid < SM_TY) {
      const int y = y0 + tid;
      const bool in = y < a.n_y;
      q_m = in ? a.row_m[y] : 0.f; q_f = in ? a.row_f[y] : -__builtin_inff(); q_u = in ? a.row_u[y] : 0.f; q_t = in ? a.targets[y] : -1;
    }
  };
  auto store_rows = [&](int buf) {
    if (PASS == 2 && tid < 64) {
      const unsigned neg = (unsigned)__builtin_amdgcn_ballot_w64(q_u < 0.f), none = (unsigned)__builtin_amdgcn_ballot_w64(q_u == 0.f);
      if (tid < SM_TY) {
        rows_m[buf][tid] = q_m; rows_f[buf][tid] = PAIRS ? q_f : q_f - q_m; rows_u[buf][tid] = q_u;
        rows_t[buf][tid] = q_u != 0.f ? q_t : -1;          // a row that no query counts for has no reference yet, and 0 times its inverse is no number
        rows_keep[buf][tid] = q_u == 0.f ? 0 : -1;
        if (tid == 0) { rows_neg[buf] = neg; rows_none[buf] = none; }
      }
    }
  };
  if (t_begin < t_end) {
    if constexpr (IMG) {
#pragma unroll
      for (int p = 0; p < NCW; ++p) copy(t_begin, 0, p);
      ask_exps(t_begin);
    } else {
#pragma unroll
      for (int w = 0; w < NSG; ++w) stage[w].begin(Y, a.y_stride, a.n_y, t_begin * SM_TY, 64 * w + tid);
      unrolled<NSG * G::NP>([&](auto k) { constexpr int w = k / G::NP, p = k % G::NP; stage[w].load(p, dim, 64 * w + tid); });
    }
    load_rows(t_begin * SM_TY);
  }

  // Pass 2: largest log2 |u| - e of the part's queries whose answer is one of the workgroup's rows.  (One array for all rows, which
  // k_loss_rows raised by atomics, held 8,192 queries with popular answers up 40 us.)
  if constexpr (PASS == 2 && REFS) {
    for (int k = tid; k < 128; k += 256) own[k] = SM_NO_OWN;
    __syncthreads();
    const int64_t first = (int64_t)stripe * 128, y_end = min((int64_t)a.n_y, (int64_t)t_end * SM_TY);
    for (int64_t y0 = (int64_t)t_begin * SM_TY; y0 < y_end; y0 += 4 * 256) {
      int id[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) { const int64_t y = y0 + 256 * k + tid; id[k] = y < y_end ? a.targets[y] : -1; }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (id[k] < first || id[k] >= first + 128) continue;
        const int64_t y = y0 + 256 * k + tid;
        const float u = a.row_u[y];
        if (u != 0.f) atomicMax(&own[id[k] - (int)first], own_key(log2f(fabsf(u)) - (PAIRS ? (float)a.yimg.exps[y >> 3] : 0.f)));
      }
    }
    __syncthreads();
  }

  // ---- stationary fragments
  v8s xh[NK], xl[PAIRS ? NK : 1];
  const int64_t x = x_first + m;
  const bool xv = x < a.n_x;
  const int64_t xr = xv ? x : a.n_x - 1;
  const T* xrow = (const T*)a.X + xr * a.x_stride;         // not for images
  int ex = 0;
  const int tgt = PASS == 1 && xv ? a.targets[xr] : -1;
  const uint32_t* words = PASS == 0 && a.allowed ? a.allowed + xr * a.allowed_stride : nullptr;
  if constexpr (IMG) {
    const int64_t xt = min(x_first / SM_TY, (int64_t)(a.n_x - 1) / SM_TY);         // the wave's rows are a tile
    const char* const row = a.ximg.tiles + xt * G::TILE + m * G::PA;
    const int swz = 16 * sp_swizzle(G::UNITS, m);
    if (PAIRS) ex = a.ximg.row_exps[32 * xt + m];
    unrolled<NK>([&](auto step) {
      constexpr int s = step;
      xh[s] = *reinterpret_cast<const v8s*>(row + ((32 * s + 16 * h) ^ swz));
      if constexpr (PAIRS) xl[s] = *reinterpret_cast<const v8s*>(row + G::PLANE + ((32 * s + 16 * h) ^ swz));
    });
  }
  if constexpr (!IMG && !PAIRS) unrolled<NK>([&](auto step) {
    constexpr int s = step;
    xh[s] = __builtin_bit_cast(v8s, load8_bits(xrow, 16 * s + 8 * h, dim));
    if (s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
  });
  if constexpr (!IMG && PAIRS) {
    // the row's exponent first, then its parts: from registers up to 128 columns (a second read is a memory latency), else read again
    constexpr bool HOLD = NK <= 8;
    float v[HOLD ? NK : 1][8];
    int big = 0;
    unrolled<NK>([&](auto step) {
      constexpr int s = step, at = HOLD ? s : 0;
      load8<TYPE>(xrow, 16 * s + 8 * h, dim, v[at]);
      if (!HOLD) {
#pragma unroll
        for (int e = 0; e < 8; ++e) big = max(big, finite_bits(v[at][e]));
        if (s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    });
    if constexpr (HOLD) {
#pragma unroll
      for (int s = 0; s < NK; ++s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) big = max(big, finite_bits(v[s][e]));
      }
    }
    big = max(big, __shfl_xor(big, 32));
    ex = sm_exponent(big);
    unrolled<NK>([&](auto step) {
      constexpr int s = step, at = HOLD ? s : 0;
      if (!HOLD) load8<TYPE>(xrow, 16 * s + 8 * h, dim, v[at]);
      sm_parts8(v[at], __builtin_ldexpf(1.f, ex), xh[s], xl[s]);
      if (!HOLD && s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    });
  }

  v16f oacc[NO];
#pragma unroll
  for (int c = 0; c < NO; ++c) oacc[c] = (v16f)(0.f);
  float ref = SM_NO_REF, lsum = 0.f, ltot = 0.f, asum = 0.f, atot = 0.f;
  // fp32 pairs in pass 1: weights follow t - e, and their sum, which is one of 2^t, would leave the floats' range where all rows are tiny
  // (e near 116): it has a reference of its own, ref - es, which moves when a score exceeds it by more than SM_SUM_ABOVE.
  int es = 0;
  if (PASS == 2 && REFS) {                                 // the weights of the row's own queries stay below it
    const int top = own[wave * 32 + m];
    if (top != SM_NO_OWN) ref = __builtin_ceilf(own_float(top)) - SM_BELOW;
  }
  unsigned word_next = PASS == 0 && a.allowed && t_begin < t_end ? words[t_begin] : ~0u;
  int group_left = a.group_tiles;
  int64_t group = PASS == 0 ? t_begin / max(a.group_tiles, 1) : 0;             // finished groups
  float first_max = SM_NO_REF, second_max = SM_NO_REF;     // of the group so far (scores before their factor k)
  v4f first4 = (v4f)(SM_NO_REF), second4 = first4;
  float neg1 = -1.f;
  asm volatile("" : "+v"(neg1));

  // ---- where a lane reads in a tile: row m, unit 2 s + h; transposed: row 16 s + 4 h + i / 4 (and 8 more), columns 32 c + 16 (g % 2) + 4 (i % 4)
  // Rows start at whole groups of units, so a unit of the same group is a bit pattern away and the other groups are immediate
  // offsets; rows y and y + 16 have the same swizzle.
  constexpr int GU = sp_group(G::UNITS);
  auto at = [](int base, int byte) { return (base ^ (byte % (16 * GU))) + byte / (16 * GU) * (16 * GU); };
  const int fofs = m * G::PA + ((16 * h) ^ (16 * sp_swizzle(G::UNITS, m)));
  const int ty = 4 * h + (i >> 2), tbyte = 32 * (g & 1) + 8 * (i & 3);
  const int trofs = ty * G::PA + (tbyte ^ (16 * sp_swizzle(G::UNITS, ty))), trofs8 = (ty + 8) * G::PA + (tbyte ^ (16 * sp_swizzle(G::UNITS, ty + 8)));
  // rare: a real branch, or it is executed speculatively; wide rows: one block at a time leaves the accumulation registers
  constexpr bool WIDE = sm_waves(TYPE, NK, PASS) == 1;
  auto rescale = [&](float f) {
    asm volatile("" : "+v"(f));
    unrolled<NO>([&](auto block) {
      constexpr int c = block;
      if (WIDE) asm volatile("" : "+a"(oacc[c]));
      oacc[c] *= f;
      if (WIDE) asm volatile("" : "+a"(oacc[c]));
    });
  };
  auto land = [&](int buf) {                               // the tile on its way is in LDS, but for the barrier
    if constexpr (IMG) {
      if (PAIRS && tid < NE) exps[buf][tid] = ye;
      store_rows(buf);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
      unrolled<NSG>([&](auto k) { constexpr int w = k; stage[w].template store<true>(smem + buf * G::TILE, nullptr, exps[buf], dim, 64 * w + tid); });
    }
  };
  if (!IMG) __syncthreads();                               // the zeros are there
  if (t_begin < t_end) land(0);
  __syncthreads();

  for (int t = t_begin; t < t_end; ++t) {
    const int buf = FEW ? 0 : (t - t_begin) & 1, bofs = buf * G::TILE;
    const int y0 = t * SM_TY;
    const bool has_next = t + 1 < t_end;                   // uniform
    unsigned word = word_next;
    if (PASS == 0 && has_next && a.allowed) word_next = words[t + 1];
    if (has_next) {
      if constexpr (IMG) ask_exps(t + 1);
      else {
#pragma unroll
        for (int w = 0; w < NSG; ++w) stage[w].begin(Y, a.y_stride, a.n_y, y0 + SM_TY, 64 * w + tid);
        // a wave of its own: all that it will want next at once
        if constexpr (FEW) unrolled<NSG * G::NP>([&](auto k) { constexpr int w = k / G::NP, p = k % G::NP; stage[w].load(p, dim, 64 * w + tid); });
      }
      load_rows(y0 + SM_TY);
    }

    // ---- scores; the streamed fragments are read PD steps ahead, the next tile's pieces are asked for between the steps
    v16f sc = (v16f)(0.f);
    {
      constexpr int PD = PAIRS ? 2 : (NK < 4 ? NK : 4);
      v8s f[PD][PL];
      const int fb = bofs + fofs;
      auto read = [&](int s) {
#pragma unroll
        for (int k = 0; k < PL; ++k) f[s % PD][k] = *reinterpret_cast<const v8s*>(smem + at(fb, 32 * s) + k * G::PLANE);
      };
#pragma unroll
      for (int s = 0; s < PD; ++s) read(s);
      unrolled<NK>([&](auto step) {
        constexpr int s = step;
        const v8s yh = f[s % PD][0], yl = f[s % PD][PL - 1];
        if (s + PD < NK) read(s + PD);
        if constexpr (PAIRS) { sc = sm_mfma<TYPE>(yl, xh[s], sc); sc = sm_mfma<TYPE>(yh, xl[s], sc); }
        sc = sm_mfma<TYPE>(yh, xh[s], sc);
        if (has_next) {
          if constexpr (IMG) {
#pragma unroll
            for (int p = s * NCW / NK; p < (s + 1) * NCW / NK; ++p) copy(t + 1, buf ^ 1, p);
          } else if constexpr (!FEW) {
#pragma unroll
            for (int p = s * G::NP / NK; p < (s + 1) * G::NP / NK; ++p) stage[0].load(p, dim, tid);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    int ey[4] = {0, 0, 0, 0};
    if (PAIRS && PASS != 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) ey[k] = __builtin_amdgcn_readfirstlane(exps[buf][k]);
    }
    // pass 0: rows scale their scores themselves, so that none, masked out or not, takes bits from another
    if constexpr (PAIRS && PASS == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int4 e4 = *reinterpret_cast<const int4*>(&exps[buf][8 * j + 4 * h]);
        const int e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[4 * j + i] = __builtin_ldexpf(sc[4 * j + i], -ex - e[i]);
      }
    }
    // ---- the first transposed fragments of the second product: step s of 16 rows, block c of 32 columns
    constexpr int NG = 2 * NO, PG = SECOND ? (PAIRS ? 2 : (NG < 4 ? NG : 4)) : 1;
    v8s tf[PG][PL];
    auto read_tr = [&](int n) {
      const int s = n / NO, c = n % NO;
#pragma unroll
      for (int k = 0; k < PL; ++k)
        tf[n % PG][k] = join8(lds_read_tr(smem + at(bofs + trofs, 64 * c) + 16 * s * G::PA + k * G::PLANE),
                              lds_read_tr(smem + at(bofs + trofs8, 64 * c) + 16 * s * G::PA + k * G::PLANE));
    };
    constexpr bool EARLY = !PAIRS && PASS == 1;            // where registers allow
    if constexpr (SECOND && EARLY) {
#pragma unroll
      for (int n = 0; n < PG; ++n) read_tr(n);
    }

    float w[16];
    bool remainder = false;                                // PASS 2, 16-bit types: own weights' remainders count too
    // ---- t = sc k[r / 4]: scores in log2 units
    float k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = PAIRS && PASS != 0 ? fmaxf(__builtin_ldexpf(a.c, max(-200, min(120, -(ex + ey[j])))), 0x1p-126f) : a.c;   // never 0: -inf times it stays
    if constexpr (PASS != 2) {
      // rows that do not count: beyond the last, or not allowed
      const int left = a.n_y - y0;
      if (left < 32) word &= (1u << left) - 1u;
      const bool some = (PASS == 0 && a.allowed) || left < 32;             // uniform
      const unsigned bits = word >> (4 * h);
      if (some) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = pick((unsigned)((int)(bits << (31 - (8 * (r >> 2) + (r & 3)))) >> 31), sc[r], -__builtin_inff());
      }
      float ztop;
      if (PASS == 0 && a.first) {                        // uniform
        // The largest and the second largest score of the lane's 16, the register's number in their lowest four bits (a score is
        // as good as known without them): the rows behind them need not be looked for.
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          v[r] = __uint_as_float((__float_as_uint(sc[r]) & ~15u) | r);
          if (some) v[r] = pick((unsigned)((int)(bits << (31 - (8 * (r >> 2) + (r & 3)))) >> 31), v[r], SM_NO_REF);   // -inf would become a NaN
        }
        float one = fmaxf(v[0], v[1]), two = fminf(v[0], v[1]);
#pragma unroll
        for (int r = 2; r < 16; ++r) { two = __builtin_amdgcn_fmed3f(one, two, v[r]); one = fmaxf(one, v[r]); }
        ztop = one;
        second_max = fmaxf(fmaxf(fminf(first_max, one), second_max), two);
        first_max = fmaxf(first_max, one);
      } else if constexpr (PAIRS && SECOND) {
        ztop = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float big = fmaxf(fmaxf(sc[4 * j], sc[4 * j + 1]), fmaxf(sc[4 * j + 2], sc[4 * j + 3])) * k[j];
          ztop = fmaxf(ztop, big - (float)ey[j]);
        }
      } else {
        ztop = sc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) ztop = fmaxf(ztop, sc[r]);
      }
      if (PASS == 0) ztop = __uint_as_float(__float_as_uint(ztop) & ~15u);   // the same reference with and without the numbers
      if (!PAIRS || PASS == 0) ztop *= k[0];
      // the reference moves
      bool moves = ztop > (PASS == 0 ? ref : ref + SM_ABOVE);
      if (PAIRS && SECOND) moves = moves || es + max(max(ey[0], ey[1]), max(ey[2], ey[3])) > (int)(SM_SUM_ABOVE - SM_ABOVE);   // t may exceed it
      if (__any(moves)) {
        if (SECOND) ztop = fmaxf(ztop, __shfl_xor(ztop, 32));              // both halves' weights meet in one product
        const float to = fmaxf(ref, SECOND ? __builtin_ceilf(ztop) - SM_BELOW : ztop), by = ref - to, fct = __builtin_amdgcn_exp2f(by);
        if (PASS == 0) {
          const float l = lsum + ltot;
          asum = l != 0.f ? fct * __builtin_fmaf(by, l, asum + atot) : 0.f;
          atot = 0.f;
        }
        float by_sum = fct;
        if constexpr (PAIRS && SECOND) {
          float ttop = -__builtin_inff();
#pragma unroll
          for (int j = 0; j < 4; ++j) ttop = fmaxf(ttop, fmaxf(fmaxf(sc[4 * j], sc[4 * j + 1]), fmaxf(sc[4 * j + 2], sc[4 * j + 3])) * k[j]);
          ttop = fmaxf(ttop, __shfl_xor(ttop, 32));
          const float from = ref - (float)es, to_sum = ttop > from + SM_SUM_ABOVE ? __builtin_ceilf(ttop) : from;
          by_sum = __builtin_amdgcn_exp2f(from - to_sum);
          es = (int)(to - to_sum);
        }
        lsum *= by_sum; ltot *= by_sum;
        if constexpr (SECOND) rescale(fct);
        ref = to;
      }
      float l16 = 0.f, a16 = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float kg = SECOND && PAIRS ? ref + (float)ey[j] : ref;
        float sum4 = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * j + e;
          float z = __builtin_fmaf(sc[r], k[j], -kg);
          if (PASS == 0 && some) z = pick((unsigned)((int)(bits << (31 - (8 * j + e))) >> 31), z, -1.0e30f);
          w[r] = __builtin_amdgcn_exp2f(z);
          sum4 += w[r];
          if (PASS == 0) a16 = __builtin_fmaf(w[r], z, a16);
        }
        l16 += SECOND && PAIRS ? __builtin_ldexpf(sum4, ey[j] + es) : sum4;
      }
      lsum += l16;
      if (PASS == 0) asum += a16;
      if ((t & (SM_CHAIN - 1)) == SM_CHAIN - 1) {        // uniform
        ltot += lsum; lsum = 0.f;
        if (PASS == 0) { atot += asum; asum = 0.f; }
      }
      if (PASS == 0 && a.first) {
        if (group_left == 1 || !has_next) {              // uniform
          const int64_t n = ++group, row = (x * 2 + h) * a.half;
          if constexpr (FEW) {                           // parts begin where it suits the table
            if (xv) { a.first[row + n - 1] = first_max; a.second[row + n - 1] = second_max; }
          } else {
            // four groups of a lane at a time: stores of 4 bytes a row apart cost as much as the products
            first4 = (v4f){first4[1], first4[2], first4[3], first_max};
            second4 = (v4f){second4[1], second4[2], second4[3], second_max};
            if (xv) {
              if ((n & 3) == 0) {
                *reinterpret_cast<v4f*>(a.first + row + n - 4) = first4;
                *reinterpret_cast<v4f*>(a.second + row + n - 4) = second4;
              } else if (!has_next) {                    // a part's last groups
#pragma unroll
                for (int j = 1; j < 4; ++j) if (j >= 4 - (int)(n & 3)) { a.first[row + n - 4 + j] = first4[j]; a.second[row + n - 4 + j] = second4[j]; }
              }
            }
          }
          first_max = second_max = SM_NO_REF;
        }
      }
      if constexpr (PASS == 1) {
        // the answer's own row is left out of the product: its weight less one may cancel, and is applied in fp32 at the end
        const int mine = tgt - y0;
        if (__any(mine >= 0 && mine < 32)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) w[r] = mine == 8 * (r >> 2) + 4 * h + (r & 3) ? 0.f : w[r];
        }
      }
    } else {
      // ---- weights p u of the tile's queries (rows) for the lane's table row
      const int tm = rows_t[buf][m];
      const bool hit = __any(tm >= x_first && tm < x_first + 32);   // the answer of one of the tile's queries is among the wave's rows
      const unsigned neg = (unsigned)__builtin_amdgcn_readfirstlane((int)rows_neg[buf]);
      float ztop = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 f4 = *reinterpret_cast<const float4*>(&rows_f[buf][8 * j + 4 * h]);
        const float fr[4] = {f4.x, f4.y, f4.z, f4.w};
        float mr[4] = {0.f, 0.f, 0.f, 0.f};
        if (PAIRS) {
          const float4 m4 = *reinterpret_cast<const float4*>(&rows_m[buf][8 * j + 4 * h]);
          mr[0] = m4.x; mr[1] = m4.y; mr[2] = m4.z; mr[3] = m4.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * j + e;
          w[r] = PAIRS ? __builtin_fmaf(sc[r], k[j], -mr[e]) + (fr[e] - (float)ey[j]) : __builtin_fmaf(sc[r], k[j], fr[e]);
          if (REFS) ztop = fmaxf(ztop, w[r]);
        }
        if (PAIRS) __builtin_amdgcn_sched_barrier(0);    // a block's statistics at a time: registers are full
      }
      if constexpr (REFS) {
        if (__any(ztop > ref + SM_ABOVE)) {
          ztop = fmaxf(ztop, __shfl_xor(ztop, 32));
          const float to = fmaxf(ref, __builtin_ceilf(ztop) - SM_BELOW), fct = __builtin_amdgcn_exp2f(ref - to);
          rescale(fct);
          ref = to;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] = __builtin_amdgcn_exp2f(REFS ? w[r] - ref : w[r]);
      if (neg) {                                         // uniform
        const unsigned bits = neg >> (4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = __uint_as_float(__float_as_uint(w[r]) ^ ((bits << (31 - (8 * (r >> 2) + (r & 3)))) & 0x80000000u));
      }
      if (hit) {                                           // an answer's own weight less u, before it is rounded
        float own_p = -1.f, f = 1.f;                       // largest own weight before, -1: none
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 u4 = *reinterpret_cast<const float4*>(&rows_u[buf][8 * j + 4 * h]);
          const int4 t4 = *reinterpret_cast<const int4*>(&rows_t[buf][8 * j + 4 * h]);
          const float u[4] = {u4.x, u4.y, u4.z, u4.w};
          const int id[4] = {t4.x, t4.y, t4.z, t4.w};
          if (REFS) f = __builtin_amdgcn_exp2f(-(ref + (float)ey[j]));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * j + e;
            const bool mine = id[e] == (int)x;
            if (!PAIRS) own_p = fmaxf(own_p, mine ? fabsf(w[r]) : -1.f);
            w[r] -= mine ? u[e] * f : 0.f;
          }
        }
        // What own weights lose to 16 bits makes a row's gradient as inexact as its own rounding does (bf16, u of any size: off by 2.6e-3
        // of its norm where that is 1.7e-3).  A weight of p - 1 with p up to 2^-10 (fp16 2^-13) loses no more than a quarter of that.
        if (!PAIRS) remainder = __any(a.weights ? own_p >= 0.f : own_p > (TYPE == MAR_DTYPE_BF16 ? 0x1p-10f : 0x1p-13f) * f);
      }
    }
    if (PASS == 0) group_left = group_left == 1 ? a.group_tiles : group_left - 1;

    // ---- O^T += Y^T P
    if constexpr (SECOND) {
      v8s ph[2], pl[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float p8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p8[e] = w[8 * s + e];
        if constexpr (PAIRS) {
          split8<true>(p8, neg1, ph[s], pl[s]);
        } else {
          ph[s] = sm_round8<TYPE>(p8);
        }
      }
      // no weight is none whatever the score: an infinite one plus log2 0 is no number
      if (PASS == 2 && __builtin_amdgcn_readfirstlane((int)rows_none[buf])) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const v8s keep = join8(*reinterpret_cast<const v4s*>(&rows_keep[buf][16 * s + 4 * h]), *reinterpret_cast<const v4s*>(&rows_keep[buf][16 * s + 8 + 4 * h]));
          ph[s] &= keep;
          if (PAIRS) pl[s] &= keep;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!EARLY) {
#pragma unroll
        for (int n = 0; n < PG; ++n) read_tr(n);
      }
      if constexpr (WIDE) unrolled<NO>([&](auto block) { constexpr int c = block; v16f& o = oacc[c]; asm volatile("" : "+a"(o)); });
      unrolled<NG>([&](auto step) {
        constexpr int n = step, s = n / NO, c = n % NO;
        const v8s yh = tf[n % PG][0], yl = tf[n % PG][PL - 1];
        if (n + PG < NG) read_tr(n + PG);
        if constexpr (PAIRS) { oacc[c] = sm_mfma<TYPE>(yl, ph[s], oacc[c]); oacc[c] = sm_mfma<TYPE>(yh, pl[s], oacc[c]); }
        oacc[c] = sm_mfma<TYPE>(yh, ph[s], oacc[c]);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (!PAIRS && PASS == 2) {
        if (remainder) unrolled<2>([&](auto half) {        // 16 of the tile's queries each
          constexpr int s = half;
          float r8[8];
          bool some = false;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int4 t4 = *reinterpret_cast<const int4*>(&rows_t[buf][16 * s + 8 * k + 4 * h]);
            const int id[4] = {t4.x, t4.y, t4.z, t4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = w[8 * s + 4 * k + e];
              r8[4 * k + e] = id[e] == (int)x ? v - sm_rounded<TYPE>(v) : 0.f;
              some = some || id[e] == (int)x;
            }
          }
          if (__any(some)) {
            const v8s rest = sm_round8<TYPE>(r8);
            unrolled<NO>([&](auto step) {
              constexpr int c = step;
              read_tr(s * NO + c);
              oacc[c] = sm_mfma<TYPE>(tf[(s * NO + c) % PG][0], rest, oacc[c]);
              __builtin_amdgcn_sched_barrier(0);
            });
          }
        });
      }
    }
    if (FEW) asm volatile("" ::: "memory");                // LDS operations of a wave complete in order
    if (has_next) land(FEW ? 0 : buf ^ 1);
    if (FEW) asm volatile("" ::: "memory"); else __syncthreads();
  }

  // ---- what the part leaves
  if (PASS == 0) {
    float l = lsum + ltot, s = asum + atot;
    sm_join(ref, l, s, __shfl_xor(ref, 32), __shfl_xor(l, 32), __shfl_xor(s, 32));
    if (h == 0 && xv) a.stats[(size_t)part * a.n_x + x] = make_float4(ref, l, s, 0.f);
  }
  if (PASS == 1) {                                       // the halves of a tile's rows share their reference
    const float lw = lsum + ltot, l = lw + __shfl_xor(lw, 32);
    if (h == 0 && xv) a.stats[(size_t)part * a.n_x + x] = make_float4(ref, l, ref - (float)es, 0.f);
  }
  if constexpr (SECOND) {
    float f = 1.f;                                       // twice the square root: the power itself may leave the floats' range
    if (PASS == 2 && REFS) f = __builtin_amdgcn_exp2f(0.5f * ref);
    const float g2 = PASS == 2 ? a.scale * f : f;          // the scale stays out of the weights: theirs of 1 are exact
    unrolled<NO>([&](auto block) {
      constexpr int c = block;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = 32 * c + 8 * j + 4 * h;
        const float v[4] = {oacc[c][4 * j] * f * g2, oacc[c][4 * j + 1] * f * g2, oacc[c][4 * j + 2] * f * g2, oacc[c][4 * j + 3] * f * g2};
        if (!xv || col >= dim) continue;
        if (PASS == 2 && a.out) store_cols<TYPE, 4>((T*)a.out + x * a.out_stride, col, dim, v);
        else *reinterpret_cast<float4*>(a.O + ((size_t)part * a.n_x + x) * a.o_pitch + col) = make_float4(v[0], v[1], v[2], v[3]);
      }
    });
  }
}

// Images of two matrices: a workgroup a tile, the first matrix's first, from tile `begin` on.
template <int TYPE, int NK>
__global__ void __launch_bounds__(256)
k_softmax_pack(SmPackArgs first, SmPackArgs second, int begin) {
  typedef SmGeom<TYPE, NK> G;
  typedef typename RowType<TYPE>::T T;
  const int tiles = (int)(((int64_t)first.n + SM_TY - 1) / SM_TY);
  const int at = begin + (int)blockIdx.x;
  const SmPackArgs a = at < tiles ? first : second;
  const int tid = threadIdx.x, t = at < tiles ? at : at - tiles, y = min(t * SM_TY + (tid >> 3), a.n - 1);
  char* const tile = a.to.tiles + (size_t)t * G::TILE;
  SmStage<TYPE, NK> stage;
  stage.begin((const T*)a.src, a.stride, a.n, t * SM_TY, tid);
#pragma unroll
  for (int p = 0; p < G::NP; ++p) stage.load(p, a.dim, tid);
  stage.apart = a.apart != 0;
  if (a.ids) {
    const int id = a.ids[y];
    if (id < 0 || id >= a.num_ids || (a.weights && fabsf(a.weights[y]) < a.least_weight)) {
      bool finite = true;
      for (int c = tid & 7; c < a.dim; c += 8) finite = finite && fabsf((float)stage.row[c]) <= 3.4028234663852886e38f;
      // the row's eight threads are neighbours, all of them here
      unsigned bad = finite ? 0u : 1u;
      bad |= __shfl_xor(bad, 1); bad |= __shfl_xor(bad, 2); bad |= __shfl_xor(bad, 4);
      stage.zero = bad != 0u;
      stage.apart = true;
    }
  }
  // units that no piece fills: up to the pitch
  for (int u = 2 * NK + (tid & 7); u < G::UNITS; u += 8) {
#pragma unroll
    for (int k = 0; k < G::PLANES; ++k)
      *reinterpret_cast<row_u4*>(tile + k * G::PLANE + (tid >> 3) * G::PA + ((16 * u) ^ (16 * sp_swizzle(G::UNITS, tid >> 3)))) = (row_u4)(0u);
  }
  stage.template store<false>(tile, a.to.exps + 4 * (size_t)t, a.to.row_exps + SM_TY * (size_t)t, a.dim, tid);
}

// Natural logarithm of a sum of weights: the exponent apart from the mantissa, whose logarithm keeps its bits, also beside 1.
__device__ __forceinline__ double log_of_sum(float l) {
  int e;
  float m = frexpf(l, &e);
  if (m < 0.70710678f) { m *= 2.f; --e; }
  return (double)e * 0.69314718055994530942 + (double)logf(m);
}
// A log probability: a score in 64 bits less a log-sum-exp of scores in 32 may come out above 0.
__device__ __forceinline__ double at_most_0(double v) { return v > 0.0 ? 0.0 : v; }   // NaN stays
