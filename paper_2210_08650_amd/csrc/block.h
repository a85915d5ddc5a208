// Internal declarations of the trained block's operators: the gradients' norm and
// clipping, rotary positions with the heads' norm, and cross attention.
#pragma once

#include "tail.h"

namespace hapi {

// ----------------------------------------------------------------- gradients

constexpr int kGradTensors = 120;   // of a launch: their addresses are its arguments (4 KB at most)
constexpr int kGradBlocks = 1024;   // of a launch, and its partial sums, at most
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
constexpr int kRotaryParts = 1024;  // partial sums of the gammas' gradients, at most

struct RotaryArgs {
  const void *x[2], *dy[2];       // of q and of k
  void *y[2];                     // forward: y; backward: dx
  const float *gamma[2];          // null: no norm
  int64_t x_st[2][3], y_st[2][3]; // batch, token, head; x: x and dx; y: y and dy
  int32_t heads[2];
  const int64_t *positions;       // [axes][tokens]
  const double *freq;             // [pairs]
  const int64_t *lens;            // [batch] or null
  float *part;                    // [blocks][2][dim]
  float *dgamma[2];
  int64_t tokens;
  int32_t len, dim, pairs, axes;
  int32_t first[kRotaryAxes];     // an axis' first pair
  int32_t head_groups;            // groups of lanes that share a token's heads
  float eps, inv_dim;
  bool norm, neighbours;
};
// Values of a pair's side that one lane handles: 16 bytes of them where all widths,
// strides and addresses allow it.
hipError_t launch_rotary_forward(bool bf16, int v, const RotaryArgs &a, hipStream_t s);
hipError_t launch_rotary_backward(bool bf16, int v, const RotaryArgs &a, hipStream_t s);

}  // namespace hapi
