// Softmax over all rows of a table (gfx950): arguments, plan and the contraction shared by log probabilities
// (mar_softmax.hip) and by the loss with its gradients (mar_softmax_loss.hip).
//
// Scores are s = scale q . w for T queries and V rows.  A pass keeps "stationary" rows in registers (32 a wave and block), streams
// the other matrix through LDS in tiles of 32 rows and takes a tile's scores with v_mfma_f32_32x32x16: A = the streamed rows from
// LDS, B = the stationary rows, so that a lane holds 16 scores of its one stationary row and no statistic crosses lanes.
//   PASS 0  stationary queries, streamed table: running reference, sum of weights and entropy sum, maxima of groups of rows
//   PASS 1  stationary queries, streamed table: the same without the entropy, and O = sum of weights times rows
//   PASS 2  stationary table rows, streamed queries: O = sum of weights times queries, with the finished log-sum-exp
// bf16 and fp16 values go to the matrix pipe as they are; an fp32 value v is v 2^e = hi + lo, both f16 (mar_split.h), a product
// three of theirs.  Exponents are the rows' own in pass 0; rows that a second product sums over (passes 1 and 2) share one by eights.
//
// Lane layouts (lane = 32 h + m = 16 g + i): A lane holds streamed row m, columns 16 s + 8 h .. + 7 of step s; B lane the same
// columns of stationary row m; D lane holds stationary row m, register r = streamed row 8 (r / 4) + 4 h + r % 4.  Second product
// O^T[c][x] += sum_y Y[y][c] P[y][x], 16 of the tile's rows a step: B = P as it lies in the registers, so slot j of half h stands for
// row 16 s + 8 (j / 4) + 4 h + j % 4; A = Y^T by the LDS transpose read (mar_split.hip describes it).
#pragma once
#include "mar_common.h"
#include "mar_split.h"

constexpr int sm_nk(int d) { return d <= 32 ? 2 : (d <= 64 ? 4 : (d <= 112 ? 7 : (d <= 128 ? 8 : (d <= 192 ? 12 : (d <= 256 ? 16 : 25))))); }
#define MAR_SOFTMAX_MAX_PARTS 64  // of the passes with a second product: a lane of k_loss_rows each
#define SM_TY 32                  // rows of a tile
#define SM_NO_REF -3.0e38f        // reference of a row that has met no score yet

// Tiles of rows as the passes read them ("images", [tiles][planes][32][pitch], units of a row in the order of sp_swizzle), with the
// exponents of every eight rows (of those that count) and of every row: laid out once, they are copied into LDS as they lie, by every
// stripe.
struct SmImage { char* tiles; int *exps, *row_exps; };       // [tiles][4], [tiles][32]

struct SmArgs {
  const void *X, *Y;               // stationary and streamed rows
  SmImage ximg, yimg;              // the same as images
  int64_t x_stride, y_stride;
  int32_t n_x, n_y, dim, nstripes, units;
  int32_t parts, tps;              // parts of the streamed tiles, tiles each
  float c, scale;                  // c = scale log2(e)
  // [parts][n_x]: reference (log2 units); sum of 2^(t - reference), in pass 1 with a reference of its own, the third number; pass 0: sum of
  // the weights times (t - reference)
  float4* stats;
  float *first, *second;           // [n_x][2][half]: largest and second largest score of a group: one half's rows of group_tiles tiles
  int64_t half;                    // groups a half, rounded up to a multiple of 4
  int32_t group_tiles;
  const uint32_t* allowed; int64_t allowed_stride;
  const int32_t* targets; const float* weights;
  float* O; int32_t o_pitch;       // [parts][n_x][o_pitch]
  const float* row_m; const float* row_f; const float* row_u;   // pass 2: per query, see k_loss_rows
  void* out; int64_t out_stride;   // pass 2 in one part: the gradient itself
};

// A weight below this counts as 0: its inverse, and the weights' reference below it, stay floats.
#define SM_LEAST_WEIGHT 0x1p-100f
// Lays rows out as images.  ids: where not NULL, a row whose id lies outside 0 .. num_ids - 1 or whose weight is below least_weight
// does not count: its exponent is its own and no other row's, and it becomes zeros if it holds values that are not finite.
struct SmPackArgs {
  const void* src; int64_t stride; int32_t n, dim;
  SmImage to;
  int32_t apart;                   // every row has an exponent of its own
  const int32_t* ids; const float* weights; int64_t num_ids;
  float least_weight;
};
static inline int64_t sm_tiles(int64_t rows) { return (rows + SM_TY - 1) / SM_TY; }
size_t sm_image_bytes(int dtype, int dim, int64_t rows);   // a multiple of 256
static inline size_t sm_exps_bytes(int64_t rows) { return ((size_t)sm_tiles(rows) * (4 + SM_TY) * 4 + 255) / 256 * 256; }
static inline SmImage sm_image(void* tiles, void* exps, int64_t rows) { return {(char*)tiles, (int*)exps, (int*)exps + 4 * sm_tiles(rows)}; }
hipError_t sm_pack(int dtype, const SmPackArgs& first, const SmPackArgs& second, hipStream_t st);   // one width

// Launches hold fewer than 2^32 threads: launch(first workgroup, workgroups) for as many launches as it takes.
constexpr int64_t sm_most_blocks(int threads) { return 0xffffffffll / threads; }
template <typename F> static inline void sm_launches(int64_t blocks, int threads, F launch) {
  for (int64_t b0 = 0; b0 < blocks; b0 += sm_most_blocks(threads)) {
    const int64_t left = blocks - b0;
    launch(b0, (unsigned)(left < sm_most_blocks(threads) ? left : sm_most_blocks(threads)));
  }
}
// Waves per query of k_loss_rows: many parts are worth several, while they make one launch.
static inline int sm_loss_waves(int parts, int64_t n) { return parts > 4 && n <= sm_most_blocks(256) ? 4 : 1; }

struct SmPlan { int32_t stripes, parts, tps, ntiles; };

const char* sm_check(const mar_softmax* p, int* code);
SmPlan sm_plan(int dtype, int dim, int pass, int mode, int64_t n_x, int64_t n_y, int multiple);
