// Launches of the AdamW step (adamw.hip).
#pragma once
#include "dla_common.h"
#include "dla_train.h"

namespace dla {

constexpr int64_t kAdamWMost = ((int64_t)1 << 36) - 4096;   // elements of a tensor

struct AdamWScalars {
  float beta1, rest1, beta2, rest2;   // rest = 1 - beta
  float lr, step_size;                // lr / (1 - beta1^step)
  float root2, eps;                   // 1 / sqrt(1 - beta2^step)
  uint32_t seed;
  const float* grad_scale;
};

hipError_t launch_adamw(const dla_adamw_tensor* t, int n, const AdamWScalars& s, int param_dtype,
                        int grad_dtype, bool f8, hipStream_t st);

}  // namespace dla
