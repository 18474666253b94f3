// Launches of the short causal convolution (short_conv.hip).
#pragma once
#include "dla_block.h"
#include "dla_common.h"

namespace dla {

struct ConvRows {
  void* p = nullptr;
  int64_t sb = 0, st = 0;
};

struct ConvArgs {
  int B, T, C, W;
  int w_f32, silu;
  const int32_t* lengths;
  const uint8_t* starts;
  const void *w, *bias, *state;
  ConvRows x, y;      // backward: y is dy
  void* state_out;    // forward
  // backward
  ConvRows dx;
  const void* dstate_out;
  void* dstate;
  float* part;        // [groups][C][W + 1], sums of dw and dbias
  // work: each sequence in `chunks` runs of `per` tokens, `lanes` pieces of a run side by side
  int per, chunks, pieces, lanes;
  int passes;         // times that a workgroup of the backward pass goes on to other runs
  int64_t groups;     // workgroups of each `lanes` pieces
};

// Fills the last line of the arguments.
void plan_conv(ConvArgs& a, int dtype, bool backward);
hipError_t launch_conv(const ConvArgs& a, int dtype, hipStream_t st);
hipError_t launch_conv_backward(const ConvArgs& a, int dtype, float* dw, float* db, hipStream_t st);

}  // namespace dla
