// Scores of queries against every row of a table in microscaled 4-bit floats, on the matrix pipe's scaled 4- and 6-bit forms (gfx950).
//
// s_ij = scale sum_b 2^(e_jb) sum_(k in b) q_ik c_jk over blocks b of 32 columns.  The table enters the products as it lies: one lane's
// 32 columns of v_mfma_scale_f32_32x32x64 are one block with its own scale.  A query in 4 bits does likewise.  Other queries are written
// block by block as slices of signed base-32 digits,  q = sum_s d_s 2^(e - 3 - 5 s),  e the exponent of the block's largest magnitude,
// |d| <= 16:  d_s / 8 is a 6-bit float (2 exponent, 3 mantissa bits) whose code is |d| with the sign, 2^(e - 5 s) its block's scale.
// Five slices hold 24 bits, counted from the block's largest value: every product is exact, sums are the matrix pipe's in fp32, smallest
// slice first.  6- and 4-bit operands run at four times the rate of 16-bit ones, so that five slices cost less than two 16-bit products,
// and the table takes a quarter of the registers that it would take in 16 bits.
//
// Blocks whose magnitudes lie far apart (wide ones, see mx_pack) lose with this what a row sees that has zeros at the large values.  What such
// blocks leave over is cut into slices again, with scales of its own, up to three times: further images.
//
// Lane layouts (lane = 32 h + m): A lane holds query m, block 2 k + h of step k; B lane the same block of table row m; D lane holds
// row m, register r = query 8 (r / 4) + 4 h + r % 4.
#include "mar_common.h"
#include "mar_flash.h"
#include "mar_mxfp.h"
#include "mar_rows_dev.h"
#include "mar_softmax.h"

typedef int mx_v8 __attribute__((ext_vector_type(8)));
typedef float mx_f16 __attribute__((ext_vector_type(16)));

#define MX_LEVELS 4                 // images of a query that may be needed
// Images of 32 queries each: [slice][step]: 16 bytes of every lane, then (6-bit slices) 8 more; then the scales of every slice, a byte a step;
// then (6-bit slices) a byte a step that says how many further images the step has.
template <int NK, int NS> struct MxImage {
  static constexpr int FRAG = NS == 1 ? 1024 : 1536, NW = (NK + 3) / 4;
  static constexpr int SCALES = NS * NK * FRAG, FURTHER = SCALES + NS * NW * 256, BYTES = (FURTHER + (NS == 1 ? 0 : 8) + 1023) / 1024 * 1024;
};
static int mx_image_bytes(int nk, int ns) { return (ns * nk * (ns == 1 ? 1024 : 1536) + ns * ((nk + 3) / 4) * 256 + (ns == 1 ? 0 : 8) + 1023) / 1024 * 1024; }
constexpr int mx_slices_of(int type) { return type == MAR_DTYPE_MXFP4 ? 1 : 5; }

struct MxArgs {
  const void* queries; const uint8_t* query_scales;
  const uint8_t *codes, *scales;
  void* out; char* images;
  int64_t query_stride, query_scales_stride, codes_stride, scales_stride, out_stride;
  int32_t n, num_rows, dim, row_blocks, out_type;
  int32_t stripes, parts, tiles_part;    // stripes of rows; parts of the queries' tiles, tiles each
  float scale;
};

// Over the four threads of a block: lanes 1 0 3 2, then 2 3 0 1.
template <typename J> __device__ __forceinline__ int mx_joined(int v, J join) {
  v = join(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false));
  return join(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false));
}
struct MxMax { __device__ __forceinline__ int operator()(int x, int y) const { return max(x, y); } };
struct MxAdd { __device__ __forceinline__ int operator()(int x, int y) const { return x + y; } };
// What remains of values o 2^unit after the slices of an image, and so on `level` times: v, the largest of the block in [8, 16) 2^20 again (or all 0), the
// new unit, and a bit for each value of which something remains.  What slices hold is o 2^grid rounded to an integer, grid that of the last
// slice, whatever the images before.
template <int NS> __device__ __forceinline__ void mx_rest(const float (&o)[8], int level, int& unit, float (&v)[8], unsigned& some) {
  for (int l = 0; l < level; ++l) {
    const int grid = unit + 5 * (NS - 1);
    int from[8], most = -10000;                            // v is v 2^from of the grid's
    some = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int x = __builtin_amdgcn_frexp_expf(o[e]) + grid;          // |o 2^grid| in [2^(x - 1), 2^x)
      const float t = __builtin_ldexpf(o[e], min(max(x, -30), 25) - __builtin_amdgcn_frexp_expf(o[e]));
      const bool small = x < -20;                          // no slice holds any of it
      v[e] = small ? o[e] : (x > 24 ? 0.f : t - rintf(t));
      from[e] = small ? grid : 0;
      if (v[e] != 0.f) { some |= 1u << e; most = max(most, __builtin_amdgcn_frexp_expf(v[e]) + from[e]); }
    }
    most = mx_joined(most, MxMax());
    const int up = most == -10000 ? 0 : 4 - most;
    unit = grid + up;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_ldexpf(v[e], from[e] + up + 20);
  }
}
// One of the 256 NK pieces of an image: eight columns of a block of one query (four neighbouring threads a block).  Its values, or four
// bytes of codes and the scale; zeros where there is no such query or block.
template <int TYPE> struct MxPiece { float v[8]; };
template <> struct MxPiece<MAR_DTYPE_MXFP4> { unsigned codes, scale; };
template <int TYPE>
__device__ __forceinline__ MxPiece<TYPE> mx_take(const MxArgs& a, int64_t q, int piece) {
  const int part = piece & 3, b = 2 * (piece >> 8) + (piece >> 7 & 1);
  const bool in = q < a.n && b < a.row_blocks;
  MxPiece<TYPE> r = {};
  if constexpr (TYPE == MAR_DTYPE_MXFP4) {
    r.scale = 127;
    if (in) {
      r.codes = *reinterpret_cast<const unsigned*>((const uint8_t*)a.queries + q * a.query_stride + 16 * b + 4 * part);
      r.scale = a.query_scales[q * a.query_scales_stride + b];
    }
  } else {
    typedef typename RowType<TYPE>::T T;
    if (in) load8<TYPE>((const T*)a.queries + q * a.query_stride, 32 * b + 8 * part, a.dim, r.v);
  }
  return r;
}
// Writes the slices of what `level` images left over of a piece.
// Returns whether the block is wide and leaves something over: a value is below 2^-22 of the largest, or half of them, eight at least, below
// 2^-6 of it, or half of them below 2^-12.  So most values of a block that is not wide keep 12 to 18 bits of their own, and none vanishes;
// 16-bit values do not leave anything over within 2^-16 (bf16) and 2^-13 (fp16).  Of steps of 64 columns and 32 queries, products of
// normal variables (two embeddings), whose magnitudes crowd at 0, have one that is wide in 100, normal variables fewer than one in 1,000.
template <int TYPE, int NK>
__device__ __forceinline__ bool mx_pack(const MxPiece<TYPE>& taken, int level, int piece, char* image) {
  constexpr int NS = mx_slices_of(TYPE);
  typedef MxImage<NK, NS> I;
  const int part = piece & 3, lane = piece >> 2 & 63, k = piece >> 8;
  uint8_t* scales = (uint8_t*)image + I::SCALES + ((k / 4) * 64 + lane) * 4 + k % 4;
  if constexpr (TYPE == MAR_DTYPE_MXFP4) {
    *reinterpret_cast<unsigned*>(image + k * 1024 + lane * 16 + 4 * part) = taken.codes;
    if (part == 0) *scales = (uint8_t)taken.scale;
    return false;
  } else {
    float o[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = taken.v[e];
    int largest = 0;
    unsigned least = ~0u;                                  // of those that are not 0, less 1
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned m = __float_as_uint(o[e]) & 0x7fffffffu;
      largest = max(largest, (int)m);
      least = min(least, m - 1);
    }
    largest = mx_joined(largest, MxMax());
    const bool finite = largest < 0x7f800000;
    const int field = max(largest >> 23, 1);
    int unit = 130 - field, below6 = 0;                    // scales are 2^(3 - unit): the block's largest is in [8, 16) times 2^-unit
    unsigned some = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!finite) o[e] = 0.f;
      v[e] = __builtin_ldexpf(o[e], unit + 20);
    }
    bool vanish = finite && field > 22 && least < ((unsigned)(field - 22) << 23) - 1u;
    if (level) {
#pragma unroll
      for (int e = 0; e < 8; ++e) some |= o[e] != 0.f ? 1u << e : 0u;
      mx_rest<NS>(o, level, unit, v, some);
      vanish = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) vanish = vanish || ((some >> e & 1u) && __builtin_fabsf(v[e]) < 2.f);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) below6 += (__float_as_uint(v[e]) & 0x7fffffffu) - 1u < 0x47ffffffu;      // 0 < |v| < 2^17
    const int votes = mx_joined(below6 + (vanish ? 0x100 : 0) + (least < ((unsigned)max(field - 12, 0) << 23) || level ? 0x10000 : 0), MxAdd());
    vanish = (votes & 0xff00) != 0;
    bool wide = vanish;
    if ((votes & 0xff) >= 8 || votes >= 0x10000) {         // few blocks: how many values there are
      int all = 0, below12 = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned m = (__float_as_uint(v[e]) & 0x7fffffffu) - 1u;
        all += m != ~0u;
        below12 += m < 0x44ffffffu;                        // 2^11
      }
      const int both = mx_joined(all + (below12 << 8), MxAdd());
      wide = wide || ((votes & 0xff) >= 8 && 2 * (votes & 0xff) >= (both & 0xff)) || (both >= 0x100 && 2 * (both >> 8) >= (both & 0xff));
    }
    // rint(v) = sum_s d_s 32^(4 - s): with 16 added to every digit they are its bits.  Four digits f = d + 16 (0 .. 32) a word, six bits each, become
    // codes together: f - 16 where f >= 16, else 16 - f with the sign 32 = (f ^ 63) + 1 - 16.
    unsigned m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = (unsigned)((int)rintf(v[e]) + 16 * 0x108421);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      unsigned c[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        unsigned x = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) x |= (s ? m[4 * half + e] >> (20 - 5 * s) & 31u : m[4 * half + e] >> 20) << (6 * e);
        const unsigned negative = ~(x >> 4 | x >> 5) & 0x041041u;
        c[half] = (x ^ ((negative << 6) - negative)) + negative - 0x410410u;
      }
      const int scale = 130 - unit - 5 * s;
      if (scale < 0) c[0] = c[1] = 0;                      // scales end at 2^-127
      char* frag = image + (s * NK + k) * I::FRAG;
      const unsigned words[3] = {c[0], c[0] >> 16 | c[1] << 8, c[1] >> 8};
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int byte = 6 * part + 2 * i;
        *reinterpret_cast<unsigned short*>(frag + (byte < 16 ? lane * 16 + byte : 1024 + lane * 8 + byte - 16)) = (unsigned short)words[i];
      }
      if (part == 0) scales[s * I::NW * 256] = (uint8_t)(finite || level ? max(scale, 0) : 255);
    }
    if (!wide) return false;
    bool over = vanish;
#pragma unroll
    for (int e = 0; e < 8; ++e) over = over || v[e] != rintf(v[e]);
    return over;
  }
}
// A workgroup a tile and step: images are laid out once and read by every stripe of rows.  999 queries of 390 columns: 5 us, bound by the launch
// and one trip to memory.  Further images are written where the step is wide.
template <int TYPE, int NK>
__global__ void __launch_bounds__(256)
k_mxfp_pack(MxArgs a) {
  typedef MxImage<NK, mx_slices_of(TYPE)> I;
  __shared__ int some[4];
  const int64_t tile = blockIdx.x / NK, tiles = (a.n + 31) / 32, q = tile * 32 + (threadIdx.x >> 2 & 31);
  const int k = (int)(blockIdx.x - tile * NK), piece = k * 256 + threadIdx.x;
  char* image = a.images + (size_t)tile * I::BYTES;
  const MxPiece<TYPE> taken = mx_take<TYPE>(a, q, piece);
  for (int level = 0; ; ++level) {
    const bool more = mx_pack<TYPE, NK>(taken, level, piece, image + (size_t)level * tiles * I::BYTES);
    if (TYPE == MAR_DTYPE_MXFP4) return;
    __syncthreads();
    const int one = __ballot(more) != 0;
    if ((threadIdx.x & 63) == 0) some[threadIdx.x >> 6] = one;
    __syncthreads();
    if (level + 1 < MX_LEVELS && __builtin_amdgcn_readfirstlane(some[0] | some[1] | some[2] | some[3])) continue;
    if (threadIdx.x == 0) image[I::FURTHER + k] = (char)level;
    return;
  }
}

// Step J of an image's products with RT x 32 rows: slice NS - 1 - J / NK, so that the smallest comes first, block pair J % NK, whose scales
// are byte J % NK % 4 of their words.  The next step's operand is read ahead of its products.
template <int NK, int NS>
__device__ __forceinline__ mx_v8 mx_operand(const char* image, int lane, int j) {
  typedef MxImage<NK, NS> I;
  const char* frag = image + ((NS - 1 - j / NK) * NK + j % NK) * I::FRAG;
  mx_v8 q = {0, 0, 0, 0, 0, 0, 0, 0};
  const row_u4 lo = *reinterpret_cast<const row_u4*>(frag + lane * 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = (int)lo[i];
  if constexpr (NS > 1) {
    const uint2 hi = *reinterpret_cast<const uint2*>(frag + 1024 + lane * 8);
    q[4] = (int)hi.x; q[5] = (int)hi.y;
  }
  return q;
}
template <int J, int NK, int NS, int RT>
__device__ __forceinline__ void mx_steps(const char* image, int lane, const mx_v8& q, const int (&qs)[NS][(NK + 3) / 4], const row_u4 (&w)[RT][NK],
                                         const int (&ws)[RT][(NK + 3) / 4], mx_f16 (&acc)[RT]) {
  if constexpr (J < NS * NK) {
    constexpr int S = NS - 1 - J / NK, K = J % NK;
    mx_v8 next = q;
    if constexpr (J + 1 < NS * NK) next = mx_operand<NK, NS>(image, lane, J + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const mx_v8 r = {(int)w[t][K][0], (int)w[t][K][1], (int)w[t][K][2], (int)w[t][K][3], 0, 0, 0, 0};
      // operand types: 2 = 6 bits (2 exponent, 3 mantissa), 4 = 4 bits
      acc[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(q, r, acc[t], NS > 1 ? 2 : 4, 4, K % 4, qs[S][K / 4], K % 4, ws[t][K / 4]);
    }
    __builtin_amdgcn_sched_barrier(0);
    mx_steps<J + 1, NK, NS, RT>(image, lane, next, qs, w, ws, acc);
  }
}

// A row's scale bytes as they are loaded, without a branch or a byte beyond the row: one or two bytes, two halves of three or four, or whole words, the
// last of the row's last four bytes; and settled: block 2 k + h in byte k % 4 of word k / 4, zeros beyond the row.
template <int NK> struct MxScales { unsigned word[NK <= 2 ? 2 : (NK + 1) / 2]; };
template <int NK> __device__ __forceinline__ MxScales<NK> mx_take_scales(const uint8_t* scales, int row_blocks) {
  MxScales<NK> r;
  if constexpr (NK == 1) { r.word[0] = scales[0]; r.word[1] = scales[row_blocks - 1]; }
  else if constexpr (NK == 2) {
    unsigned short half[2];
    __builtin_memcpy(&half[0], scales, 2);
    __builtin_memcpy(&half[1], scales + row_blocks - 2, 2);
    r.word[0] = half[0]; r.word[1] = half[1];
  } else {
#pragma unroll
    for (int j = 0; j < (NK + 1) / 2; ++j) __builtin_memcpy(&r.word[j], scales + min(4 * j, row_blocks - 4), 4);
  }
  return r;
}
template <int NK>
__device__ __forceinline__ void mx_settle_scales(const MxScales<NK>& taken, int row_blocks, int h, int (&ws)[(NK + 3) / 4]) {
  constexpr int ND = (NK + 1) / 2;
  unsigned d[ND + 1];
  if constexpr (NK == 1) d[0] = row_blocks == 1 ? taken.word[0] : taken.word[0] | taken.word[1] << 8;
  else if constexpr (NK == 2) d[0] = taken.word[0] | (taken.word[1] >> (8 * (4 - row_blocks))) << 16;
  else {
#pragma unroll
    for (int j = 0; j < ND; ++j) d[j] = taken.word[j] >> (8 * max(4 * j + 4 - row_blocks, 0));         // by less than 32: there are more than 4 j blocks
  }
  d[ND] = 0u;
  const unsigned pick = h ? 0x07050301u : 0x06040200u;
#pragma unroll
  for (int k = 0; k < (NK + 3) / 4; ++k) ws[k] = (int)__builtin_amdgcn_perm(d[2 * k + 1], d[2 * k], pick);
}
// A wave's 32 RT rows of the table, lane m's RT neighbours from row0 on, block 2 k + h.  Rows beyond the last are taken for it and not written.
template <int NK, int RT>
__device__ __forceinline__ void mx_load_rows(const MxArgs& a, int row0, int h, row_u4 (&w)[RT][NK], int (&ws)[RT][(NK + 3) / 4]) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t row = min(row0 + t, a.num_rows - 1);
    const uint8_t* codes = a.codes + row * a.codes_stride;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int b = 2 * k + h;
      w[t][k] = (row_u4)(0u);
      if (b < a.row_blocks) w[t][k] = *reinterpret_cast<const row_u4*>(codes + 16 * b);
    }
    mx_settle_scales<NK>(mx_take_scales<NK>(a.scales + row * a.scales_stride, a.row_blocks), a.row_blocks, h, ws[t]);
  }
}
// The same of 32 RT rows from `first` on, 32 t + m, with loads of 64 bytes of a row where two steps remain: sixteen lanes take block 0 (of
// four) of rows 0 .. 15, the next block 2, then 1 and 3; another load the same of rows 16 .. 31.  mx_settle exchanges lanes 16 .. 31 and
// 48 .. 63 of the first with lanes 0 .. 15 and 32 .. 47 of the second, which leaves a step in each.  Nothing waits for a load here, and no lane
// goes without: where a row has no such block its last one is taken, which meets zeros (1 query, 4,000,000 x 400: 235 us with branches
// and scales taken apart at once, 185 so).
template <int NK, int RT>
__device__ __forceinline__ void mx_fetch_rows(const MxArgs& a, int first, int lane, row_u4 (&w)[RT][NK], MxScales<NK> (&taken)[RT]) {
  const int m = lane & 31, h = lane >> 5, i = lane & 15, block = (lane >> 5) | (lane >> 4 & 1) << 1;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t row = min((int64_t)first + 32 * t + m, (int64_t)a.num_rows - 1);
    taken[t] = mx_take_scales<NK>(a.scales + row * a.scales_stride, a.row_blocks);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t last = a.num_rows - 1, row = min((int64_t)first + 32 * t + m, last);
    const uint8_t* low = a.codes + min((int64_t)first + 32 * t + i, last) * a.codes_stride;
    const uint8_t* high = a.codes + min((int64_t)first + 32 * t + 16 + i, last) * a.codes_stride;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const bool pair = k + 1 < NK || k % 2;
      const uint8_t* const codes = pair ? (k % 2 ? high : low) : a.codes + row * a.codes_stride;
      w[t][k] = *reinterpret_cast<const row_u4*>(codes + 16 * min(pair ? 4 * (k / 2) + block : 2 * k + h, a.row_blocks - 1));
    }
  }
}
template <int NK, int RT>
__device__ __forceinline__ void mx_settle(const MxArgs& a, int h, row_u4 (&w)[RT][NK], const MxScales<NK> (&taken)[RT], int (&ws)[RT][(NK + 3) / 4]) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    mx_settle_scales<NK>(taken[t], a.row_blocks, h, ws[t]);
#pragma unroll
    for (int k = 0; k + 1 < NK; k += 2)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const auto r = __builtin_amdgcn_permlane16_swap(w[t][k][d], w[t][k + 1][d], false, false);
        w[t][k][d] = r[0]; w[t][k + 1][d] = r[1];
      }
  }
}

// All slices of an image, the smallest first.
template <int NK, int NS, int RT>
__device__ __forceinline__ void mx_tile(const char* image, int lane, const row_u4 (&w)[RT][NK], const int (&ws)[RT][(NK + 3) / 4], mx_f16 (&acc)[RT]) {
  typedef MxImage<NK, NS> I;
  int qs[NS][I::NW];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
#pragma unroll
    for (int k = 0; k < I::NW; ++k) qs[s][k] = *reinterpret_cast<const int*>(image + I::SCALES + ((s * I::NW + k) * 64 + lane) * 4);
  }
  mx_steps<0, NK, NS, RT>(image, lane, mx_operand<NK, NS>(image, lane, 0), qs, w, ws, acc);
}
// Step K of further image `level`, out of memory, where the step has one.
template <int K, int NK, int NS, int RT>
__device__ __forceinline__ void mx_further(const char* image, unsigned long long further, int level, int lane, const row_u4 (&w)[RT][NK],
                                           const int (&ws)[RT][(NK + 3) / 4], mx_f16 (&acc)[RT]) {
  if constexpr (K < NK) {
    typedef MxImage<NK, NS> I;
    if ((int)(further >> (8 * K) & 255) >= level) {        // uniform
#pragma unroll
      for (int s = NS - 1; s >= 0; --s) {
        const mx_v8 q = mx_operand<NK, NS>(image, lane, (NS - 1 - s) * NK + K);
        const int scale = *reinterpret_cast<const int*>(image + I::SCALES + ((s * I::NW + K / 4) * 64 + lane) * 4);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const mx_v8 r = {(int)w[t][K][0], (int)w[t][K][1], (int)w[t][K][2], (int)w[t][K][3], 0, 0, 0, 0};
          acc[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(q, r, acc[t], 2, 4, K % 4, scale, K % 4, ws[t][K / 4]);
        }
      }
    }
    mx_further<K + 1, NK, NS, RT>(image, further, level, lane, w, ws, acc);
  }
}

// Scores of 32 queries from `q0` on, below n, and a lane's RT neighbouring rows: a wave instruction writes two queries' 32 RT scores.  Where these do not begin
// with lines of 128 bytes a large result takes up to 1.4 times as long (325 x 679,723 x 27 in fp32: 183 us, rows at multiples of 64 bytes 212, at
// odd places 261; neighbouring stripes on one die do not change that): a lane holds one row for all queries, whose rows lie differently.
template <int TYPE, int RT>
__device__ __forceinline__ void mx_store(const MxArgs& a, int64_t q0, int64_t n, int row0, int h, bool whole, const mx_f16 (&acc)[RT]) {
  typedef typename RowType<TYPE>::T T;
  T* const base = (T*)a.out + (q0 + 4 * h) * a.out_stride + row0;
  T* next = base;
  // Sixteen masks and multiples of the stride, kept from call to call, would be more than the scalar registers hold: found anew.
  int64_t stride = a.out_stride;
  int left = (int)min(n - q0, (int64_t)32) - 4 * h;
  if (!whole) { asm volatile("" : "+s"(stride)); asm volatile("" : "+v"(left)); }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int i = 8 * (r / 4) + r % 4;
    T* const to = whole ? base + i * a.out_stride : next;
    next += r % 4 == 3 ? 5 * stride : stride;
    T v[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) v[t] = (T)(acc[t][r] * a.scale);
    if (whole) { __builtin_memcpy(to, v, sizeof(v)); continue; }
    if (q0 + i >= n) break;                              // uniform: half 0's queries come first
    if (i < left) {
#pragma unroll
      for (int t = 0; t < RT; ++t) if (row0 + t < a.num_rows) to[t] = v[t];
    }
  }
}
template <int RT>
__device__ __forceinline__ void mx_store_any(const MxArgs& a, int64_t q0, int64_t n, int row0, int h, bool whole, const mx_f16 (&acc)[RT]) {
  if (a.out_type == MAR_DTYPE_FP32) { if (whole) mx_store<0, RT>(a, q0, n, row0, h, true, acc); else mx_store<0, RT>(a, q0, n, row0, h, false, acc); }
  else if (a.out_type == MAR_DTYPE_BF16) { if (whole) mx_store<1, RT>(a, q0, n, row0, h, true, acc); else mx_store<1, RT>(a, q0, n, row0, h, false, acc); }
  else { if (whole) mx_store<2, RT>(a, q0, n, row0, h, true, acc); else mx_store<2, RT>(a, q0, n, row0, h, false, acc); }
}

// Many queries: eight waves hold 32 RT rows each and take the images out of LDS, G at a time; the next G are copied there meanwhile.  Rows
// stay, since 4 bits of a row take a tenth of the registers that a query's slices would: with four rows a lane, 24 bytes of an image serve
// four products.
// 999 fp32 queries, 120,007 x 390: 131 to 157 us, 3.2 to 3.9 TB/s and 3.4 to 4.1 PFLOP/s of slices' products (matrix pipe busy 47 % at 1.9 GHz,
// no bank conflicts); 4,096 in 4 bits, 131,072 x 400 to bf16: 167 to 190 us, 5.7 to 6.4 TB/s of scores,
// which bound it.  What bounds the
// first: writing a tile's scores and forming the next's take turns in a wave, two waves a SIMD cover each other in part; products as dense
// as 4,096 16-bit queries of 400 columns with 131,072 rows (485 to 515 us; 420 to 445 with four slices, whose 19 bits cut 16-bit values off) are
// bound by power.  Further images are read out of memory, not staged: 999 x 120,007 x 390 with an outlier of 2^12 in one column takes 1.35
// times as long, with one in every block 2.4 times.
template <int NK, int NS> constexpr int mx_group() { return MxImage<NK, NS>::BYTES > 16 * 1024 ? 1 : 32 * 1024 / MxImage<NK, NS>::BYTES; }
template <int NK, int NS, int RT>
__global__ void __launch_bounds__(512)
k_mxfp_scores(MxArgs a) {
  typedef MxImage<NK, NS> I;
  constexpr int G = mx_group<NK, NS>(), STAGE = G * I::BYTES;
  __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  const int part = (int)blockIdx.x / a.stripes, stripe = (int)blockIdx.x - part * a.stripes;
  const int first = (stripe * 8 + wave) * 32 * RT, row0 = first + (lane & 31) * RT;
  const int tiles = (a.n + 31) / 32, t0 = part * a.tiles_part, t1 = min(tiles, t0 + a.tiles_part);
  // images t .. t + G - 1, those that there are, by loads that write LDS, 1 KB a wave instruction.  In asm: the compiler would have
  // every read of LDS wait for them, of the other half too
  int token = 0;
  auto copy = [&](int t, int buf) {
    const int bytes = min(G, t1 - t) * I::BYTES;
    const v4i words = buf_words(a.images + (size_t)t * I::BYTES, (uint32_t)bytes);
    const unsigned to = (unsigned)(unsigned long long)(__attribute__((address_space(3))) const char*)smem + buf * STAGE;
    for (int at = wave * 1024; at < bytes; at += 8 * 1024) buf_load4_to_lds(words, to + at, lane * 16, at, token);
  };
  copy(t0, 0);
  row_u4 w[RT][NK];
  int ws[RT][I::NW];
  mx_load_rows<NK, RT>(a, row0, h, w, ws);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int t = t0, buf = 0; t < t1; t += G, buf ^= 1) {
    if (t + G < t1) copy(t + G, buf ^ 1);
    const int here = min(G, t1 - t);
    for (int g = 0; g < here; ++g) {
      mx_f16 acc[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[r] = (mx_f16)(0.f);
      const char* image = smem + buf * STAGE + g * I::BYTES;
      uint2 words = make_uint2(0, 0);
      if constexpr (NS > 1) words = *reinterpret_cast<const uint2*>(image + I::FURTHER);
      mx_tile<NK, NS, RT>(image, lane, w, ws, acc);
      if constexpr (NS > 1) {                              // behind the products: before them they would wait for the word
        const unsigned long long further = ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)words.y) << 32 |
                                            (unsigned)__builtin_amdgcn_readfirstlane((int)words.x)) & ~0ull >> (64 - 8 * NK);
        if (further != 0) for (int level = 1; level < MX_LEVELS; ++level)
          mx_further<0, NK, NS, RT>(a.images + ((size_t)level * tiles + t + g) * I::BYTES, further, level, lane, w, ws, acc);
      }
      // the copies have landed; the last tile's scores need not have: nothing waits for them at the barrier
      if (g == here - 1) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int64_t q0 = (int64_t)(t + g) * 32;
      mx_store_any<RT>(a, q0, a.n, row0, h, first + 32 * RT <= a.num_rows && q0 + 32 <= a.n, acc);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
}

// Up to 32 queries: every workgroup lays out their image for itself and its waves go through the table, the next rows on their way.  Bound
// by reading the table: 1 query, 4,000,000 x 100: 50 us, 288 MB at 5.8 TB/s (a part out of the last-level cache); 4,000,000 x 400: 185 to 190 us, 884 MB
// at 4.7; 14,951 x 75: 5.2 us, a launch and two trips to memory.  The pieces of the queries that there are, not of 32, are laid out: 1 query,
// 66,000 x 400: 8 us, 17 where every workgroup goes through the places of 32.
// Where a block is wide the image holds eight queries, four images of each in the places of 32, whose sums are joined before they are written: up to
// eight queries take no more than the sums' time for it (1 query, 1,000,000 x 400: 41 and 59 us), others go through the table once for every eight (32 of
// them: 88 and 226 us).
template <int TYPE, int NK, int RT>
__global__ void __launch_bounds__(256)
k_mxfp_few(MxArgs a) {
  constexpr int NS = mx_slices_of(TYPE);
  typedef MxImage<NK, NS> I;
  __shared__ __attribute__((aligned(16))) char image[I::BYTES];
  __shared__ int some[4];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  row_u4 w[RT][NK], next[RT][NK];
  MxScales<NK> scales[RT], next_s[RT];
  const int stripe0 = (int)blockIdx.x * 4 + wave, row0 = min(stripe0, a.stripes - 1) * 32 * RT;
  mx_fetch_rows<NK, RT>(a, row0, tid & 63, w, scales);
  // pieces of the queries that there are, 2^shift >= a.n places a block, the next one's values on their way
  const int shift = a.n > 1 ? 32 - __builtin_clz(a.n - 1) : 0, pieces = 8 * NK << shift;
  auto piece_of = [&](int i) { const int block = i >> (2 + shift); return (block >> 1) * 256 + (block & 1) * 128 + (i & ((4 << shift) - 1)); };
  MxPiece<TYPE> taken = mx_take<TYPE>(a, piece_of(min(tid, pieces - 1)) >> 2 & 31, piece_of(min(tid, pieces - 1)));
  if (shift < 5) {                                         // zeros for the others
    for (int at = tid * 16; at < I::BYTES; at += 256 * 16) *reinterpret_cast<row_u4*>(image + at) = (row_u4)(0u);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
  bool more = false;
#pragma unroll 1
  for (int i = tid; i < pieces; i += 256) {
    const MxPiece<TYPE> now = taken;
    const int following = piece_of(min(i + 256, pieces - 1));
    taken = mx_take<TYPE>(a, following >> 2 & 31, following);
    more |= mx_pack<TYPE, NK>(now, 0, piece_of(i), image);
  }
  if constexpr (NS > 1) { const int one = __ballot(more) != 0; if ((tid & 63) == 0) some[wave] = one; }
  __syncthreads();
  int wide = 0;                                            // a scalar: as a truth value it would be held for every lane
  if constexpr (NS > 1) wide = __builtin_amdgcn_readfirstlane(some[0] | some[1] | some[2] | some[3]);
  for (int q0 = 0; ; q0 += 8) {
    int at = tid;
    asm volatile("" : "+v"(at));                           // the loop's addresses are not kept in registers from turn to turn
    const int lane = at & 63, h = lane >> 5, m = lane & 31;
    if constexpr (NS > 1) if (wide) {
      __syncthreads();                                     // nobody reads the image before
#pragma unroll 1
      for (int k = 0; k < NK; ++k) mx_pack<TYPE, NK>(mx_take<TYPE>(a, q0 + (at >> 2 & 7), k * 256 + at), at >> 5 & 3, k * 256 + at, image);
      __syncthreads();
      mx_fetch_rows<NK, RT>(a, row0, lane, w, scales);         // anew: no registers hold them meanwhile
    }
    const int n = wide ? min(a.n, q0 + 8) : a.n;
    int stripe = stripe0;
    while (stripe < a.stripes) {
      const int first = stripe * 32 * RT;
      stripe += (int)gridDim.x * 4;
      // behind the last stripe too where there are many: a branch here has these rows waited for at once (1 query, 4,000,000 x 100: 61 us with, 50
      // without); where a wave has one stripe alone it saves the loads (14,951 x 75: 4.9 and 5.4)
      if (RT > 1 || stripe < a.stripes) mx_fetch_rows<NK, RT>(a, min(stripe, a.stripes - 1) * 32 * RT, lane, next, next_s);
      int ws[RT][I::NW];
      mx_settle<NK, RT>(a, h, w, scales, ws);
      mx_f16 acc[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) acc[t] = (mx_f16)(0.f);
      mx_tile<NK, NS, RT>(image, lane, w, ws, acc);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {                      // a choice, no branch: that would hold all sums twice
          const float all = acc[t][r] + (acc[t][4 + r] + (acc[t][8 + r] + acc[t][12 + r]));
          acc[t][r] = wide ? all : acc[t][r];
        }
        mx_store_any<1>(a, q0, n, first + 32 * t + m, h, false, reinterpret_cast<const mx_f16 (&)[1]>(acc[t]));
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int k = 0; k < NK; ++k) w[t][k] = next[t][k];
        scales[t] = next_s[t];
      }
    }
    if (!wide || q0 + 8 >= a.n) return;
  }
}

// ------------------------------------------------------------------------------------------ launches -----
template <int TYPE, int NK> static void launch_type(const MxPlan& plan, const MxArgs& a, hipStream_t st) {
  constexpr int NS = mx_slices_of(TYPE);
  const dim3 grid((unsigned)plan.grid);
  if (plan.few) {
    if (plan.rt == 1) hipLaunchKernelGGL((k_mxfp_few<TYPE, NK, 1>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_mxfp_few<TYPE, NK, (NK <= 3 ? 4 : 2)>), grid, dim3(256), 0, st, a);
    return;
  }
  hipLaunchKernelGGL((k_mxfp_pack<TYPE, NK>), dim3((unsigned)(mx_tiles(a.n) * NK)), dim3(256), 0, st, a);
  if (plan.rt == 4) hipLaunchKernelGGL((k_mxfp_scores<NK, NS, 4>), grid, dim3(512), 0, st, a);
  else if (plan.rt == 2) hipLaunchKernelGGL((k_mxfp_scores<NK, NS, 2>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((k_mxfp_scores<NK, NS, 1>), grid, dim3(512), 0, st, a);
}
template <int NK> static void launch_nk(int dtype, const MxPlan& plan, const MxArgs& a, hipStream_t st) {
  if (dtype == MAR_DTYPE_FP32) launch_type<0, NK>(plan, a, st);
  else if (dtype == MAR_DTYPE_BF16) launch_type<1, NK>(plan, a, st);
  else if (dtype == MAR_DTYPE_FP16) launch_type<2, NK>(plan, a, st);
  else launch_type<3, NK>(plan, a, st);
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
  const int slices = mx_slices_of(p->dtype);
  const size_t bytes = (size_t)mx_tiles(p->num_queries) * (slices == 1 ? 1 : MX_LEVELS) * mx_image_bytes((p->dim + 63) / 64, slices);
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
    case 1: launch_nk<1>(p->dtype, plan, a, st); break;
    case 2: launch_nk<2>(p->dtype, plan, a, st); break;
    case 3: launch_nk<3>(p->dtype, plan, a, st); break;
    case 4: launch_nk<4>(p->dtype, plan, a, st); break;
    case 5: launch_nk<5>(p->dtype, plan, a, st); break;
    case 6: launch_nk<6>(p->dtype, plan, a, st); break;
    default: launch_nk<7>(p->dtype, plan, a, st); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { mar_set_error("score kernel: %s", hipGetErrorString(e)); return MAR_EHIP; }
  return MAR_OK;
}
