// Internal declarations of the trained block's operators: the gradients' norm and
// clipping, rotary positions with the heads' norm, and cross attention.
#pragma once

#include "tail.h"

namespace hapi {

// ----------------------------------------------------------------- gradients

constexpr int kGradTensors = 120;   // of a launch: their addresses are its arguments (4 KB at most)
constexpr int kGradBlocks = 1024;   // of a launch, and its partial sums, at most; 2048 were slower
constexpr int kGradSumLaunches = 4; // partial sums of as many launches are joined by the blocks that need them

struct GradArgs {
  const void *in[kGradTensors];
  void *out[kGradTensors];
  int64_t size[kGradTensors];
  int32_t seg[kGradTensors + 1];    // a tensor's first segment
  uint32_t f32[(kGradTensors + 31) / 32];
  int32_t count;
  int32_t seg_size;                 // values of a segment
  double *part;                     // norm: of this launch's blocks; clip: all of them
  int64_t parts;
  double max_norm;
  float *norm;                      // clip: written by the first launch, else null
};
static_assert(sizeof(GradArgs) <= 4096, "a launch's arguments");
hipError_t launch_grad_squares(const GradArgs &a, int blocks, hipStream_t s);
hipError_t launch_grad_clip(const GradArgs &a, int blocks, hipStream_t s);
// part[0 .. parts) to out (up to kGradBlocks sums); norm: the root of all of them.
hipError_t launch_grad_join(const double *part, int64_t parts, double *out, hipStream_t s);
hipError_t launch_grad_norm(const double *part, int64_t parts, float *norm, hipStream_t s);

// -------------------------------------------------------------------- rotary

constexpr int kRotaryMaxDim = 256;
constexpr int kRotaryAxes = 4;
constexpr int kRotaryParts = 512;  // partial sums of either gamma's gradient, at most

struct RotaryArgs {
  const void *x[2], *dy[2];       // of q and of k
  void *y[2];                     // forward: y; backward: dx
  const float *gamma[2];          // null: no norm
  int64_t x_st[2][3], y_st[2][3]; // batch, token, head; x: x and dx; y: y and dy
  int32_t heads[2];
  const int64_t *positions;       // [axes][tokens]
  const double *freq;             // [pairs]
  const int64_t *lens;            // [batch] or null
  float *part;                    // [2][blocks][dim]
  float *dgamma[2];
  int64_t tokens;
  int32_t len, dim, pairs, axes;
  int32_t first[kRotaryAxes];     // an axis' first pair
  int32_t head_groups[2];         // groups of lanes that share a token's heads
  float eps, inv_dim;
  bool norm, neighbours;
};
// v: values of a pair's side that one lane handles, 16 bytes of them where the widths divide
// into them and the call is large enough, at their elements' alignment.
hipError_t launch_rotary_forward(bool bf16, int v, const RotaryArgs &a, hipStream_t s);
hipError_t launch_rotary_backward(bool bf16, int v, const RotaryArgs &a, hipStream_t s);

// ----------------------------------------------------------- cross attention

constexpr int kAttendMaxDim = 128;
constexpr int kAttendMaxGroup = 512;  // query heads of a key head

// The rows of one key head's problem are its query heads' tokens: row r is token
// r / group, head r % group of the group.
struct AttendArgs {
  const void *q, *k, *v, *o, *dout;  // as the kernels read them: 16-byte aligned rows (o: whole 16-byte slots)
  int64_t q_st[3], k_st[3], v_st[3], o_st[3], g_st[3];  // elements; g: of dout
  void *y, *dq, *dk, *dv;            // y: o as it is written
  int64_t y_st[3], dq_st[3], dk_st[3], dv_st[3];
  int32_t y_vec, dq_vec, dk_vec, dv_vec;  // 1: four values can be stored at once; 2: 16 bytes; 4: two values
  float2 *stats;                     // [batch][q_len][heads] (largest score, log of the sum)
  const int64_t *q_lens, *kv_lens;
  const uint8_t *mask;               // [batch][kv_len] or null
  int32_t q_len, kv_len, heads, kv_heads, group, dim;
  int32_t pairs;                     // batch * kv_heads
  float scale, c;                    // c = scale log2(e)
  int32_t splits;                    // of the keys (dk, dv: of the rows) over workgroups
  float *part;                       // [splits][pairs][rows][dim4]; dk, dv: [splits][2][pairs][kv_len][dim4]
  float4 *part_ml;                   // [splits][pairs][rows] (reference score, sum about it, largest score)
  int32_t dim4;                      // dim up to a multiple of 4
  float *delta;                      // [pairs][rows] sum of dout o
};

// A workgroup's waves have 4 x 32, 2 x 32 or 32 rows between them: no more than there are
// (4 x 32 always: forward 128 x 64 x 197, 12 heads of 64, 26.7 for 24.9 us, 16 x 1 x 8192, 16 +
// 4 heads of 128, 40.1 for 38.8; 4 x 8 x 2000, 8 + 2 heads of 96, 9.3 for 10).
inline int attend_row_waves(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }
// Up to four waves in all: those that share rows take other keys, in tiles of their own,
// two of them in flight; 64 KB of the LDS, so that a CU runs two workgroups (one wave alone:
// the forward cases above 26.4 and 41.1 us, dq of 1 x 1 x 8192 16.8 for 13.5).
constexpr int attend_key_waves(int esz, int padded_dim, int row_waves) {
  const int fit = 65536 / (4 * 32 * padded_dim * esz), most = 4 / row_waves;
  return fit < 1 ? 1 : fit < most ? (fit == 3 ? 2 : fit) : most;
}
// 64 keys of 16 bits to a tile where the LDS then holds them twice, 32 of 32 bits.
constexpr int attend_tile_keys(int esz, int padded_dim, int key_waves) {
  return esz == 2 && key_waves * 4 * 64 * padded_dim * esz <= (key_waves > 1 ? 32768 : 65536) ? 64 : 32;
}
// Rows from any layout to [batch][tokens][heads][ld], zeros from dim on.
struct StageArgs {
  const void *in;
  void *out;
  int64_t st[3];
  int64_t count;  // rows
  int32_t tokens, heads, dim, ld;
};
hipError_t launch_attend_stage(bool bf16, const StageArgs &a, hipStream_t s);
hipError_t launch_attend_forward(bool bf16, const AttendArgs &a, hipStream_t s);
hipError_t launch_attend_dq(bool bf16, const AttendArgs &a, hipStream_t s);   // delta, too
hipError_t launch_attend_dkv(bool bf16, const AttendArgs &a, hipStream_t s);
// Whether P and dS of bf16 heads are multiplied with both halves, them as they are rounded
// and what the rounding left.  Over a large call the two roundings leave 1.4 times what the
// output's own does; a single row of few keys may be off by more, and a small call is all
// such rows (213 rows x 2 heads x 9 keys: dq off by 1.5 times as much as by its rounding
// alone, now 1.0 times).  So it is the call's rows that count, not the row's own sizes, and a
// row's last bits differ between a call of 512 rows and one of more.  Few rows are few
// products: 8 heads x 50 x 600 of 64 values 18 us with either, 16 x 1 x 4096, 16 heads
// of 64, 105 against 111 us, of 128, 460 against 536 us.
inline bool attend_fine(const AttendArgs &a) { return (int64_t)a.pairs * a.group * a.q_len <= 512; }
// All three in one kernel: bf16 heads of up to 64 values whose rows a workgroup's waves have
// between them, a workgroup for each group of heads.  dq's kernel and dk's and dv's form
// the scores twice, but split a group's keys over workgroups where groups are few.  Measured,
// their time against this one's: 1536 groups x 64 rows x 197 keys 79 against 57 us, 4 groups
// 17 against 13 us, 192 groups x 2048 keys 79 against 69 us, 128 groups x 4096 keys 98
// against 125 us, 64 groups x 2048 keys 41 against 64 us.  So it is taken where neither
// kernel would split, and from 192 groups on.
inline bool attend_few_rows(bool bf16, const AttendArgs &a) {
  const int64_t rows = (int64_t)a.q_len * a.group;
  return bf16 && a.dim <= 64 && rows > 0 && rows <= 64 && a.kv_len > 0;
}
hipError_t launch_attend_few_rows(const AttendArgs &a, hipStream_t s);

}  // namespace hapi
