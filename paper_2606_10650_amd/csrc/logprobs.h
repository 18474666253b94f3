// Launches of the log probabilities of rows of logits (logprobs.hip).
#pragma once
#include "dla_block.h"
#include "dla_common.h"

namespace dla {

struct LogprobArgs {
  int64_t rows;
  int V, top;
  const void* l;
  int64_t st;
  const int64_t* tokens;
  float *lp, *lse, *ent;   // backward: read
  int64_t* ids;
  float* tops;
  // backward
  const float *dlp, *dent, *dlse;
  void* dl;
  int64_t dst;
};

hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t st);
hipError_t launch_logprobs_backward(const LogprobArgs& a, int dtype, hipStream_t st);

}  // namespace dla
