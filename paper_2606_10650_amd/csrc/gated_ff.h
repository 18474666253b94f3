// Launches of the gated feed-forward block (gated_ff.hip, gated_ff_gemm.hip).
#pragma once
#include "dla_block.h"
#include "dla_common.h"

namespace dla {

struct FfRows {
  void* p = nullptr;
  int64_t st = 0;   // elements from row to row
};

// A few rows, straight from the inputs as they lie: y, and g and u where those have a place.
constexpr int kFfStepRows = 64;
hipError_t launch_ff_step(int64_t rows, int D, int F, int dtype, FfRows x, FfRows wg, FfRows wu, FfRows y, FfRows g,
                          FfRows u, hipStream_t st);

// Rows of `cols` values as bfloat16 rows of round_up(cols, 8), zeros behind the last: of bfloat16 one
// plane, of float32 three, their terms from the largest down, each plane rows round_up(cols, 8) long.
// Up to three sets of rows at once.
struct FfPack {
  int64_t rows = 0;
  int cols = 0;
  FfRows from;
  uint16_t* to = nullptr;
};
struct FfPacks {
  FfPack set[3];
};
hipError_t launch_ff_pack(const FfPacks& sets, int dtype, hipStream_t st);

// dg and du from g and u, float32, and dy: planes as above of rows with round_up(F, 8) values of dg, then as
// many of du.
hipError_t launch_ff_parts(int64_t rows, int F, int dtype, FfRows g, FfRows u, FfRows dy, uint16_t* to, hipStream_t st);

// Products of bfloat16 matrices, whose rows start at multiples of 16 bytes, summed in float32:
//   kind 0: C = sum over pairs of A B^T, A [M][K], B [N][K]; twice, with B and B2, and as y, g and u
//   kind 1: C = sum over pairs of A B, A [M][K], B [K][N]
//   kind 2: C = sum over pairs of A^T B, A [K][M], B [K][N]
// A pair names a plane of A and one of B.
constexpr int kFfPlanes = 6;
struct FfGemm {
  int kind, out_f32, pairs;
  int64_t M, N, K;
  const uint16_t* a[kFfPlanes];
  const uint16_t* b[kFfPlanes];
  const uint16_t* b2[kFfPlanes];
  int64_t lda, ldb;
  uint64_t ia, ib;    // four bits a pair, the first in the lowest
  FfRows c, g, u;     // kind 0: c is y; g and u are float32
  FfRows c2;          // kind 2: where the rows from `half` on go; each half has `rows` of them
  int64_t half, rows;
  float* part;        // FfPlan's part_bytes
};

// Who works on what: the first `full` tiles of C have a workgroup each, the rest `share`, which divide the
// steps of a tile's sum among them, and whose parts are joined afterwards.
struct FfPlan {
  int large;                // tiles of 256 x 256, or of 128 x 128
  int tiles_m, tiles_n, share;
  int64_t tiles, full, steps;
  size_t part_bytes;
  // the first step of a part
  __host__ __device__ int64_t begin(int part) const { return steps * part / share; }
};
FfPlan plan_ff_gemm(int kind, int64_t M, int64_t N, int64_t K, int pairs);
hipError_t launch_ff_gemm(const FfGemm& p, const FfPlan& w, hipStream_t st);

}  // namespace dla
