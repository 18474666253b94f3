// Launches of the norm with gate, residual sum and next norm (gated_norm.hip).
#pragma once
#include "dla_block.h"
#include "dla_common.h"

namespace dla {

struct GroupRows {
  void* p = nullptr;
  int64_t st = 0, sg = 0;
};

struct GatedNormArgs {
  int64_t rows;
  int G, D;
  float eps, scale;
  const void *w, *w2;
  int w_f32, per_group;
  GroupRows x, gate, res, h, y;   // backward: h is dh, y is dy
  float *rstd, *rstd2;
  // backward
  GroupRows dx, dgate, dres;
  float *dw_part, *dw2_part;      // [parts][dw's size], [parts][D]
  // work: workgroups side by side over groups, and along the rows
  int gcols;
  int64_t groups;
};

// Fills the last lines of the arguments.  Of the backward pass with gate and next norm these are no larger than
// without.
void plan_gated_norm(GatedNormArgs& a, int dtype, bool backward);
// Parts of dw and of dw2 of a backward pass, in floats.
int64_t gated_norm_dw_parts(const GatedNormArgs& a);
hipError_t launch_gated_norm(const GatedNormArgs& a, int dtype, bool backward, hipStream_t st);
hipError_t launch_gated_norm_dw(const GatedNormArgs& a, float* dw, float* dw2, hipStream_t st);

}  // namespace dla
