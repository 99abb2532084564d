// The contraction of mar_softmax.h on the device.
#pragma once
#include "mar_rows_dev.h"
#include "mar_softmax.h"
#include "mar_split_dev.h"

// Stationary blocks of 32 rows a wave takes.
constexpr int sm_qb(int type, int nk, int pass) { return 1; }
constexpr int sm_waves(int type, int nk, int pass) { return nk <= 8 ? 2 : (nk <= 12 && pass == 0 ? 2 : 1); }

template <int TYPE> __device__ __forceinline__ v16f sm_mfma(v8s a, v8s b, v16f c) {
  if (TYPE == MAR_DTYPE_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  return mfma32h(a, b, c);
}
// Largest finite magnitude's bits.
__device__ __forceinline__ int finite_bits(float v) { const int b = __float_as_int(v) & 0x7fffffff; return b < 0x7f800000 ? b : 0; }
// Exponent of a row or block whose largest finite magnitude has these bits: 2^e max lies in [2^14, 2^15).  Zeros take 80: the second
// product's weights are 2^(t - e), and one far from the others' exponents would leave the floats' range.
__device__ __forceinline__ int sm_exponent(int max_bits) { return max_bits == 0 ? 80 : min(141 - (max_bits >> 23), 116); }
__device__ __forceinline__ void sm_parts8(const float (&v)[8], float scale, v8s& hi, v8s& lo) {
  v8h h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) { _Float16 a, b; sp_parts(v[e] * scale, a, b); h[e] = a; l[e] = b; }
  hi = __builtin_bit_cast(v8s, h); lo = __builtin_bit_cast(v8s, l);
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

// A tile on its way from memory to LDS: wave w takes rows 8 w .. 8 w + 7.
template <int TYPE, int NK> struct SmStage {
  typedef SmGeom<TYPE, NK> G;
  typedef typename RowType<TYPE>::T T;
  row_u4 r[G::NP][G::PLANES];
  // use: where not NULL, rows with a 0 there are taken as zeros whatever they hold
  __device__ __forceinline__ void load(const T* __restrict__ Y, int64_t stride, int n_y, int dim, int y0, int tid, const float* __restrict__ use = nullptr) {
    const T* row = Y + (int64_t)min(y0 + (tid >> 3), n_y - 1) * stride;      // rows beyond the last are the last again
#pragma unroll
    for (int p = 0; p < G::NP; ++p) {
      const int u = (tid & 7) + 8 * p;
      if (TYPE == MAR_DTYPE_FP32) {
        float v[8];
        load8<TYPE>(row, 8 * u, dim, v);
        r[p][0] = (row_u4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        r[p][G::PLANES - 1] = (row_u4){__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
      } else {
        r[p][0] = load8_bits(row, 8 * u, dim);
      }
    }
    if (use && use[min(y0 + (tid >> 3), n_y - 1)] == 0.f) {
#pragma unroll
      for (int p = 0; p < G::NP; ++p) r[p][0] = r[p][G::PLANES - 1] = (row_u4)(0u);
    }
  }
  // exps: the exponents of the tile's four blocks of eight rows (fp32)
  __device__ __forceinline__ void store(char* tile, int* exps, int tid) {
    const int row = tid >> 3;
    char* const at = tile + row * G::PA;
    const int swz = 16 * sp_swizzle(G::UNITS, row);
    if (TYPE == MAR_DTYPE_FP32) {
      int big = 0;
#pragma unroll
      for (int p = 0; p < G::NP; ++p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) big = max(big, finite_bits(__uint_as_float(r[p][j >> 2 ? G::PLANES - 1 : 0][j & 3])));
      }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) big = max(big, __shfl_xor(big, o));
      const int e = sm_exponent(big);
      if ((tid & 63) == 0) exps[tid >> 6] = e;
      const float scale = __builtin_ldexpf(1.f, e);
#pragma unroll
      for (int p = 0; p < G::NP; ++p) {
        const int u = (tid & 7) + 8 * p;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r[p][j >> 2 ? G::PLANES - 1 : 0][j & 3]);
        v8s hi, lo;
        sm_parts8(v, scale, hi, lo);
        if (u < 2 * NK) {
          *reinterpret_cast<v8s*>(at + ((16 * u) ^ swz)) = hi;
          *reinterpret_cast<v8s*>(at + G::PLANE + ((16 * u) ^ swz)) = lo;
        }
      }
    } else {
#pragma unroll
      for (int p = 0; p < G::NP; ++p) {
        const int u = (tid & 7) + 8 * p;
        if (u < 2 * NK) *reinterpret_cast<row_u4*>(at + ((16 * u) ^ swz)) = r[p][0];
      }
    }
  }
};

// Softmax weights in fp16 (and as pairs of f16) lie between 2^-24 and 2^16: the reference is put 12 below the largest exponent met
// and moves when one exceeds it by more than 15; what is 2^-36 of the largest weight is lost to the second product (never to the sum).
#define SM_ABOVE 15.f
#define SM_BELOW 12.f

template <int TYPE, int NK, int PASS>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sm_waves(TYPE, NK, PASS))))
k_softmax(SmArgs a) {
  typedef SmGeom<TYPE, NK> G;
  typedef typename RowType<TYPE>::T T;
  constexpr bool PAIRS = TYPE == MAR_DTYPE_FP32;
  constexpr int QB = sm_qb(TYPE, NK, PASS);
  constexpr bool SECOND = PASS != 0;
  constexpr int NO = SECOND ? (NK + 1) / 2 : 1;            // 32-column blocks of the output
  constexpr bool REFS = PASS != 2 || TYPE != MAR_DTYPE_BF16;   // weights relative to a reference
  __shared__ __attribute__((aligned(1024))) char smem[2 * G::TILE];
  __shared__ int exps[2][4];
  __shared__ __attribute__((aligned(16))) float rows_m[2][SM_TY], rows_f[2][SM_TY], rows_u[2][SM_TY];
  __shared__ int rows_t[2][SM_TY];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, m = lane & 31, g = lane >> 4, i = lane & 15;
  // workgroups of one part of the streamed rows share an XCD's L2: XCD j takes a contiguous eighth of the (part, stripe) units
  const int unit = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  if (unit >= a.units) return;
  const int part = unit / a.nstripes, stripe = unit - part * a.nstripes;
  const int ntiles_all = (int)(((int64_t)a.n_y + SM_TY - 1) / SM_TY);
  const int t_begin = part * a.tps, t_end = min(ntiles_all, t_begin + a.tps);
  const int64_t x_first = (int64_t)stripe * (128 * QB) + wave * (32 * QB);
  const int dim = a.dim;

  // zeros: units beyond the columns that a tile's copies write
  for (int k = tid * 16; k < 2 * G::TILE; k += 256 * 16) *reinterpret_cast<row_u4*>(smem + k) = (row_u4)(0u);
  SmStage<TYPE, NK> stage;
  const T* Y = (const T*)a.Y;
  // pass 2: statistics of the tile's queries, row threadIdx.x of the first 32
  float q_m = 0.f, q_f = 0.f, q_u = 0.f;
  int q_t = -1;
  auto load_rows = [&](int y0) {
    if (PASS == 2 && tid < SM_TY) {
      const int y = y0 + tid;
      const bool in = y < a.n_y;
      q_m = in ? a.row_m[y] : -SM_NO_REF; q_f = in ? a.row_f[y] : (REFS ? -__builtin_inff() : 0.f); q_u = in ? a.row_u[y] : 0.f; q_t = in ? a.targets[y] : -1;
    }
  };
  auto store_rows = [&](int buf) {
    if (PASS == 2 && tid < SM_TY) { rows_m[buf][tid] = q_m; rows_f[buf][tid] = q_f; rows_u[buf][tid] = q_u; rows_t[buf][tid] = q_t; }
  };
  if (t_begin < t_end) { stage.load(Y, a.y_stride, a.n_y, dim, t_begin * SM_TY, tid, PASS == 2 ? a.row_u : nullptr); load_rows(t_begin * SM_TY); }

  // ---- stationary fragments
  v8s xh[QB][NK], xl[QB][PAIRS ? NK : 1];
  int ex[QB], tgt[QB];
  bool xv[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int64_t x = x_first + 32 * b + m;
    xv[b] = x < a.n_x;
    const int64_t xr = xv[b] ? x : a.n_x - 1;
    const T* row = (const T*)a.X + xr * a.x_stride;
    ex[b] = 0;
    tgt[b] = PASS == 1 && xv[b] ? a.targets[xr] : -1;
    if (PAIRS) {
      int big = 0;
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        float v[8];
        load8<TYPE>(row, 16 * s + 8 * h, dim, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) big = max(big, finite_bits(v[e]));
      }
      big = max(big, __shfl_xor(big, 32));
      ex[b] = sm_exponent(big);
    }
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      if constexpr (PAIRS) {
        float v[8];
        load8<TYPE>(row, 16 * s + 8 * h, dim, v);
        sm_parts8(v, __builtin_ldexpf(1.f, ex[b]), xh[b][s], xl[b][s]);
      } else {
        xh[b][s] = __builtin_bit_cast(v8s, load8_bits(row, 16 * s + 8 * h, dim));
      }
    }
  }

  v16f oacc[QB][NO];
  float ref[QB], lsum[QB], asum[QB], gmax[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
#pragma unroll
    for (int c = 0; c < NO; ++c) oacc[b][c] = (v16f)(0.f);
    ref[b] = SM_NO_REF; lsum[b] = asum[b] = 0.f; gmax[b] = -__builtin_inff();
  }
  float neg1 = -1.f;
  asm volatile("" : "+v"(neg1));

  // ---- where a lane reads in a tile: row m, unit 2 s + h; transposed: row 16 s + 4 h + i / 4 (and 8 more), columns 32 c + 16 (g % 2) + 4 (i % 4)
  const int fswz = 16 * sp_swizzle(G::UNITS, m), fofs = m * G::PA;
  // O^T += Y^T P.  rest: bits of the weights whose remainder after rounding to 16 bits counts too (PASS 2: of an answer's own row)
  auto second = [&](const char* tile, int b, const float (&w)[16], bool with_rest, unsigned rest) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float p8[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p8[e] = w[8 * s + e];
      v8s ph, pl = {0, 0, 0, 0, 0, 0, 0, 0};
      if constexpr (PAIRS) {
        split8<true>(p8, neg1, ph, pl);
      } else {
        ph = sm_round8<TYPE>(p8);
        if (PASS == 2 && with_rest) {
          float r8[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) r8[e] = (rest >> (8 * s + e) & 1u) ? p8[e] - sm_rounded<TYPE>(p8[e]) : 0.f;
          pl = sm_round8<TYPE>(r8);
        }
      }
      const int ty = 16 * s + 4 * h + (i >> 2), tswz = 16 * sp_swizzle(G::UNITS, ty), tswz8 = 16 * sp_swizzle(G::UNITS, ty + 8);
#pragma unroll
      for (int c = 0; c < NO; ++c) {
        const int byte = 64 * c + 32 * (g & 1) + 8 * (i & 3);
        const char* const p0 = tile + ty * G::PA + (byte ^ tswz);
        const char* const p1 = tile + (ty + 8) * G::PA + (byte ^ tswz8);
        const v8s yh = join8(lds_read_tr(p0), lds_read_tr(p1));
        oacc[b][c] = sm_mfma<TYPE>(yh, ph, oacc[b][c]);
        if constexpr (PAIRS) {
          const v8s yl = join8(lds_read_tr(p0 + G::PLANE), lds_read_tr(p1 + G::PLANE));
          oacc[b][c] = sm_mfma<TYPE>(yl, ph, oacc[b][c]);
          oacc[b][c] = sm_mfma<TYPE>(yh, pl, oacc[b][c]);
        } else if (PASS == 2 && with_rest) {
          oacc[b][c] = sm_mfma<TYPE>(yh, pl, oacc[b][c]);
        }
      }
    }
  };
  __syncthreads();                                         // the zeros are there
  if (t_begin < t_end) { stage.store(smem, exps[0], tid); store_rows(0); }
  __syncthreads();

  for (int t = t_begin; t < t_end; ++t) {
    const int buf = (t - t_begin) & 1;
    const char* const tile = smem + buf * G::TILE;
    const int y0 = t * SM_TY;
    const bool has_next = t + 1 < t_end;
    if (has_next) { stage.load(Y, a.y_stride, a.n_y, dim, y0 + SM_TY, tid, PASS == 2 ? a.row_u : nullptr); load_rows(y0 + SM_TY); }

    v16f sc[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) sc[b] = (v16f)(0.f);
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const v8s yh = *reinterpret_cast<const v8s*>(tile + fofs + ((32 * s + 16 * h) ^ fswz));
      if constexpr (PAIRS) {
        const v8s yl = *reinterpret_cast<const v8s*>(tile + G::PLANE + fofs + ((32 * s + 16 * h) ^ fswz));
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          sc[b] = sm_mfma<TYPE>(yl, xh[b][s], sc[b]); sc[b] = sm_mfma<TYPE>(yh, xl[b][s], sc[b]); sc[b] = sm_mfma<TYPE>(yh, xh[b][s], sc[b]);
        }
      } else {
#pragma unroll
        for (int b = 0; b < QB; ++b) sc[b] = sm_mfma<TYPE>(yh, xh[b][s], sc[b]);
      }
    }
    int ey[4] = {0, 0, 0, 0};
    if (PAIRS) {
#pragma unroll
      for (int k = 0; k < 4; ++k) ey[k] = __builtin_amdgcn_readfirstlane(exps[buf][k]);
    }

#pragma unroll
    for (int b = 0; b < QB; ++b) {
      // ---- t = sc k[r / 4]: scores in log2 units
      float k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = PAIRS ? fmaxf(__builtin_ldexpf(a.c, max(-200, min(120, -(ex[b] + ey[j])))), 0x1p-126f) : a.c;   // never 0: -inf times it stays
      const int64_t x = x_first + 32 * b + m;
      if (PASS != 2) {
        // rows that do not count: beyond the last, or not allowed
        const int left = a.n_y - y0;
        unsigned word = left >= 32 ? ~0u : (1u << left) - 1u;
        if (PASS == 0 && a.allowed) word &= a.allowed[min(x, (int64_t)a.n_x - 1) * a.allowed_stride + t];
        const bool some = PASS == 0 && a.allowed ? true : left < 32;     // uniform
        word >>= 4 * h;
        if (some) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[b][r] = pick((unsigned)((int)(word << (31 - (8 * (r >> 2) + (r & 3)))) >> 31), sc[b][r], -__builtin_inff());
        }
        float top = -__builtin_inff(), ztop = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float big = fmaxf(fmaxf(sc[b][4 * j], sc[b][4 * j + 1]), fmaxf(sc[b][4 * j + 2], sc[b][4 * j + 3])) * k[j];
          top = fmaxf(top, big);
          ztop = fmaxf(ztop, SECOND && PAIRS ? big - (float)ey[j] : big);
        }
        gmax[b] = fmaxf(gmax[b], top);
        // the reference moves
        if (__any(ztop > ref[b] + SM_ABOVE)) {
          ztop = fmaxf(ztop, __shfl_xor(ztop, 32));        // both halves' weights meet in one product
          const float to = fmaxf(ref[b], ztop - SM_BELOW), by = ref[b] - to, f = __builtin_amdgcn_exp2f(by);
          if (PASS == 0 && lsum[b] != 0.f) asum[b] = f * __builtin_fmaf(by, lsum[b], asum[b]);
          lsum[b] *= f;
          if (SECOND) {
#pragma unroll
            for (int c = 0; c < NO; ++c) {
#pragma unroll
              for (int r = 0; r < 16; ++r) oacc[b][c][r] *= f;
            }
          }
          ref[b] = to;
        }
        float w[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float kg = SECOND && PAIRS ? ref[b] + (float)ey[j] : ref[b];
          float sum4 = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * j + e;
            float z = __builtin_fmaf(sc[b][r], k[j], -kg);
            if (PASS == 0 && some) z = pick((unsigned)((int)(word << (31 - (8 * j + e))) >> 31), z, -1.0e30f);
            w[r] = __builtin_amdgcn_exp2f(z);
            sum4 += w[r];
            if (PASS == 0) asum[b] = __builtin_fmaf(w[r], z, asum[b]);
          }
          lsum[b] += SECOND && PAIRS ? __builtin_ldexpf(sum4, ey[j]) : sum4;
        }
        if (PASS == 0 && a.gmax) {
          const bool last = t + 1 == t_end || (t + 1) % a.group_tiles == 0;    // uniform
          if (last) {
            if (xv[b]) a.gmax[x * a.ngroups + 2 * (int64_t)(t / a.group_tiles) + h] = gmax[b];
            gmax[b] = -__builtin_inff();
          }
        }
        if constexpr (PASS == 1) {
          // the answer's own row is left out of the product: its weight less one may cancel, and is applied in fp32 at the end
          const int own = tgt[b] - y0;
          if (__any(own >= 0 && own < 32)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) w[r] = own == 8 * (r >> 2) + 4 * h + (r & 3) ? 0.f : w[r];
          }
          second(tile, b, w, false, 0u);
        }
      } else {
        // ---- weights p u of the tile's queries (rows) for the lane's table row
        float w[16];
        const int tm = rows_t[buf][m];
        const bool hit = __any(tm >= x_first + 32 * b && tm < x_first + 32 * b + 32);   // the answer of a query is among the wave's rows
        unsigned own = 0u;
        if (hit) {
#pragma unroll
          for (int r = 0; r < 16; ++r) own |= (int64_t)rows_t[buf][8 * (r >> 2) + 4 * h + (r & 3)] == x ? 1u << r : 0u;
        }
        if (!REFS) {
          // f = u / (sum of the query's weights); an answer's own weight less u, before it is rounded
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int y = 8 * (r >> 2) + 4 * h + (r & 3);
            w[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][r], k[0], -rows_m[buf][y])) * rows_f[buf][y];
          }
          if (hit) {
#pragma unroll
            for (int r = 0; r < 16; ++r) if (own >> r & 1u) w[r] -= rows_u[buf][8 * (r >> 2) + 4 * h + (r & 3)];
          }
        } else {
          // f = log2 |u| - log2(sum); weights are |p u| relative to the row's reference
          float ztop = -__builtin_inff();
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int y = 8 * (r >> 2) + 4 * h + (r & 3);
            w[r] = __builtin_fmaf(sc[b][r], k[r >> 2], -rows_m[buf][y]) + rows_f[buf][y] - (float)ey[r >> 2];
            ztop = fmaxf(ztop, w[r]);
          }
          if (hit) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              if (own >> r & 1u) ztop = fmaxf(ztop, __builtin_amdgcn_logf(fabsf(rows_u[buf][8 * (r >> 2) + 4 * h + (r & 3)])) - (float)ey[r >> 2]);
            }
          }
          if (__any(ztop > ref[b] + SM_ABOVE)) {
            ztop = fmaxf(ztop, __shfl_xor(ztop, 32));
            const float to = fmaxf(ref[b], ztop - SM_BELOW), f = __builtin_amdgcn_exp2f(ref[b] - to);
#pragma unroll
            for (int c = 0; c < NO; ++c) {
#pragma unroll
              for (int r = 0; r < 16; ++r) oacc[b][c][r] *= f;
            }
            ref[b] = to;
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float u = rows_u[buf][8 * (r >> 2) + 4 * h + (r & 3)];
            w[r] = __builtin_amdgcn_exp2f(w[r] - ref[b]);
            w[r] = u < 0.f ? -w[r] : w[r];
            if (hit && (own >> r & 1u)) {
              // |u| 2^-(ey + reference) in two steps: neither factor leaves the floats' range alone
              w[r] -= __builtin_ldexpf(u * __builtin_amdgcn_exp2f(-ref[b]), -ey[r >> 2]);
            }
          }
        }
        second(tile, b, w, hit, own);
      }
    }
    if (has_next) { stage.store(smem + (buf ^ 1) * G::TILE, exps[buf ^ 1], tid); store_rows(buf ^ 1); }
    __syncthreads();
  }

  // ---- what the part leaves
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int64_t x = x_first + 32 * b + m;
    if (PASS != 2) {                                       // the halves of a tile's rows share their reference
      const float l = lsum[b] + __shfl_xor(lsum[b], 32), s = asum[b] + __shfl_xor(asum[b], 32);
      if (h == 0 && xv[b]) a.stats[(size_t)part * a.n_x + x] = make_float4(ref[b], l, s, 0.f);
    }
    if constexpr (SECOND) {
      float f = 1.f;                                       // twice the square root: the power itself may leave the floats' range
      if (PASS == 2 && REFS) f = __builtin_amdgcn_exp2f(0.5f * ref[b]);
#pragma unroll
      for (int c = 0; c < NO; ++c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = 32 * c + 8 * j + 4 * h;
          const float v[4] = {oacc[b][c][4 * j] * f * f, oacc[b][c][4 * j + 1] * f * f, oacc[b][c][4 * j + 2] * f * f, oacc[b][c][4 * j + 3] * f * f};
          if (!xv[b] || col >= dim) continue;
          if (PASS == 2 && a.out) store_cols<TYPE, 4>((T*)a.out + x * a.out_stride, col, dim, v);
          else *reinterpret_cast<float4*>(a.O + ((size_t)part * a.n_x + x) * a.o_pitch + col) = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
    }
  }
}
