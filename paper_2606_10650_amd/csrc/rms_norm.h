// Launches of the root-mean-square norm (rms_norm.hip).
#pragma once
#include "dla_common.h"

namespace dla {

struct NormRows {
  void* p = nullptr;
  int64_t st = 0;   // elements from row to row
  // the rows from one on, of elements of the given size
  NormRows from(int64_t row, int elem) const {
    NormRows r = *this;
    if (p) r.p = static_cast<char*>(p) + row * st * elem;
    return r;
  }
};

struct NormArgs {
  int64_t rows;
  int D;
  float eps;
  const void* w;
  int w_f32;
  // forward: x, residual, h = x + residual, y; backward: dx, dres, h, dy
  NormRows x, res, h, y;
  float* rstd;
  float* y_scale;
  float* dw_part;   // [groups][D]
  int groups;
};

int norm_threads(int64_t rows, int pieces);
int norm_groups(int64_t rows, int pieces);
// kind 0: forward; 1: forward with 8-bit output; 2: backward
hipError_t launch_norm(const NormArgs& a, int dtype, int kind, hipStream_t st);
hipError_t launch_norm_dw(const NormArgs& a, float* dw, hipStream_t st);

}  // namespace dla
