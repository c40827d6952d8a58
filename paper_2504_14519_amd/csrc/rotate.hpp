// Argument block and launchers of the norm and rotation of queries and keys (internal to the library).
#pragma once
#include "kernels.hpp"

namespace slimpipe {

// One side of a call: the queries or the keys.
struct RotateSide {
  const __bf16* x;               // [batch, rows, heads, head_dim]
  const float* weight;           // [head_dim]; nullptr: ones
  __bf16* out;                   // forward: the result; backward: the gradient of x, at the strides of x
  const void* d_out;             // backward: gradient of the result, at the out strides
  int32_t d_out_f32, heads;      // heads = 0: this side is not part of the call
  int64_t stride_b, stride_s, stride_h, out_stride_b, out_stride_s, out_stride_h;
};

struct RotateArgs {
  RotateSide side[2];            // queries, keys
  const double* frequency;       // [rotate_dim / 2], radians a position
  const int64_t* positions;      // [batch, rows], or nullptr: position + row
  int64_t position;
  int32_t rows, interleaved, rotate_dim;
  float eps;
  int64_t total_rows;            // batch * rows
  // A wave takes a block of rows (64 / (head_dim / 16)) and heads_wave heads of one side, a workgroup four such blocks; backward: every wave_blocks-th
  // block from its first one on
  int32_t heads_wave, sets[2];   // sets of heads of the queries, of the keys
  int64_t row_blocks, wave_blocks;
  int32_t workgroups;            // a multiple of the sets of both
  float* part;                   // backward: sums of the weights' gradients, [workgroup][head_dim]; nullptr: not wanted
  float* d_weight[2];
  int32_t weight_accumulate;
};

constexpr int rotate_rows_per_wave(int head_dim) { return 64 / (head_dim / 16); }
// most heads of a wave: what its registers hold of loads under way
constexpr int kRotateFwdHeads = 4, kRotateBwdHeads = 4;
hipError_t launch_rotate_fwd(const RotateArgs& a, int head_dim, hipStream_t st);
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, hipStream_t st);

}  // namespace slimpipe
