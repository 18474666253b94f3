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
  int bf16;
  // work: each row in `parts` of `per` logits, and what these leave: [rows][parts][3], [rows][parts][top]
  int parts, per;
  float* part_sums;
  uint64_t* part_keys;
  // backward
  const float *dlp, *dent, *dlse;
  void* dl;
  int64_t dst;
};

// Fills parts and per.
void plan_logprobs(LogprobArgs& a, int dtype);
hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t st);
hipError_t launch_logprobs_backward(const LogprobArgs& a, int dtype, hipStream_t st);

}  // namespace dla
