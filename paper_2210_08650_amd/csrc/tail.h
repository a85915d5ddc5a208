// Internal declarations of the trained tail's operators: layer norm, and the
// cross entropy and distillation losses of a linear classifier.
#pragma once

#include "internal.h"

namespace hapi {

constexpr int64_t kMaxLaunchThreads = UINT32_MAX;  // the threads of a launch are a 32-bit number
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------- layer norm

constexpr int kNormMaxDim = 16384;
constexpr int kNormParts = 512;  // partial sums of gamma's and beta's gradients, at most

struct NormArgs {
  const void *x, *dy;
  const float *gamma, *beta;
  void *y, *dx;
  float *mean, *rstd;   // forward: written; backward: read
  float *part;          // [parts][2][dim]
  float *dgamma, *dbeta;
  int64_t rows, x_ld, y_ld;  // y_ld: of y and dy; x_ld: of x and dx
  int dim;
  float eps;
};
// Blocks of the forward kernel, which walk the rows in a stride of the grid, for `want`
// blocks' rows.
int64_t norm_forward_blocks(int64_t want, int threads);
hipError_t launch_norm_forward(bool bf16, const NormArgs &a, hipStream_t s);
hipError_t launch_norm_backward(bool bf16, const NormArgs &a, hipStream_t s);

// ------------------------------------------------------ classifier and losses

// Sparse target distribution of a row: `top` classes ids[n][k] with weights.
// Cross entropy: top = 1, ids = the targets, the weight is 1.  Distillation:
// softmax of teacher[n][k] / T over the entries with id >= 0.
struct HeadArgs {
  const void *x, *w;        // [rows][x_ld], [classes][w_ld]: k contiguous, as the products read them
  const void *x_in, *w_in;  // the caller's, any alignment
  int64_t x_ld, w_ld, x_in_ld, w_in_ld;
  const float *bias;        // [classes] or null
  const int64_t *ids;       // [rows][top]
  const float *teacher;     // [rows][top]; null: cross entropy
  int64_t rows, classes;
  int dim, top;
  float inv_t, t;           // 1 / T and T
  // forward
  float2 *part;             // [parts][rows] (max, sum of exp) of a row over a part's classes
  int parts;
  float *loss, *picked;
  float2 *stats;            // [rows] (largest logit m, log sum exp((z - m) / T))
  // backward
  const float *dloss;
  float2 *info;             // [rows_pad] (m, coefficient / sum of exp); rows that do not count: (inf, 0)
  float *unit;              // what dz^T's coefficients are divided by, in [1, 2)
  int32_t *id32;            // [rows][top] the targets' classes, -1: none
  float *cq;                // [rows][top] what they take off dz: coefficient times weight
  void *gt;                 // [piece][rows_pad] dz^T of one piece of the classes
  int64_t rows_pad, v0, piece;  // the piece is classes [v0, v0 + piece)
  float *db_part;           // [db_parts][classes], null: no bias gradient
  int db_parts;
  float *dx_part;           // [splits][rows][dx_pad]
  int splits, dx_pad;
  bool first;               // first piece
  bool dx_whole;            // one split and one piece: no partial sums
  float *dw_part;           // [w_splits][classes][dx_pad], one piece only
  int w_splits;
  int bias_slices;          // distillation of any rows: parts of dbias for what the targets take off; else 0
  void *dx, *dw;
  int64_t dx_ld, dw_ld;
  float *dbias;
};

// Tiles of the products, out of a rule on the sizes: 256 x 256, 128 x 128, 64 x 64,
// 32 rows by 128 classes (the weights stream past), 32 x 32.
enum Variant { BIG, MID, SMALL, FEW, TINY };
constexpr int64_t kCus = 256;  // compute units the rules count on
Variant head_variant(bool bf16, int64_t rows, int64_t classes);
// BIG: the classes that 256 x 256 tiles take; 128 x 128 ones take the others.
int64_t head_big_classes(int64_t rows, int64_t classes);
// The parts the forward product writes of a row, and dz's of a class.
int head_parts(bool bf16, int64_t rows, int64_t classes);
int head_db_parts(bool bf16, int64_t rows, int64_t classes);
// The forward product's launch that begins at class c0: its tiles and classes, its first
// part, and the parts there are from that one on.
struct HeadLaunch {
  Variant v;
  int64_t classes;
  int part, parts;
};
HeadLaunch head_forward_launch(bool bf16, int64_t rows, int64_t classes, int64_t c0);
// FEW: whether dx and dW are launches of their own; the splits of either product's k.
bool head_few_apart(int dim, int64_t piece);
int head_w_splits(bool bf16, int64_t rows, int dim, int64_t classes, int64_t piece);
int head_splits(bool bf16, int64_t rows, int dim, int64_t classes, int64_t piece, int w_splits);
constexpr int kBiasClasses = 128;  // classes of a block that sums dbias
int head_bias_slices(int64_t classes);
constexpr int kHeadRowPad = 64;
// FEW, and what calls of so few rows do more: bf16 dz has a second half that the first
// one's rounding left, in columns [kFewRows, 2 kFewRows) of dz^T.
constexpr int kFewRows = 32;
static_assert(2 * kFewRows <= kHeadRowPad, "both halves in the padded rows");
constexpr int kHeadPiece = 256;  // pieces are multiples of this many classes

// rows of T values from ld_in to a padded, aligned [rows][ld_out], zero from dim on.
hipError_t launch_head_stage(bool bf16, const void *in, int64_t ld_in, void *out, int64_t ld_out, int64_t rows, int dim,
                             hipStream_t s);
hipError_t launch_head_forward(bool bf16, const HeadArgs &a, hipStream_t s);  // parts
hipError_t launch_head_finish(bool bf16, const HeadArgs &a, hipStream_t s);   // loss, stats, picked
// info, id32, cq and a copy of x (xs, [rows][xs_ld]) whose rows that do not count are zero.
hipError_t launch_head_prepare(bool bf16, const HeadArgs &a, void *xs, int64_t xs_ld, hipStream_t s);
hipError_t launch_head_dlogits(bool bf16, const HeadArgs &a, hipStream_t s);  // gt, db_part; targets' entries put in
hipError_t launch_head_grads(bool bf16, const HeadArgs &a, hipStream_t s);    // dw of the piece, dx_part
hipError_t launch_head_reduce(bool bf16, const HeadArgs &a, hipStream_t s);   // dx, dbias

}  // namespace hapi
