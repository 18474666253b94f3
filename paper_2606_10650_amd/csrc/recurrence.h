// Launches of the single-state recurrence and its backward pass (recurrence.hip,
// recurrence_grad.hip, recurrence_step.hip).
#pragma once
#include "dla_common.h"
#include "dla_train.h"

namespace dla {

// Rows of one tensor: element (b, h, t, i) lies at p + b sb + (h / hdiv) sh + t st + i,
// in elements.
struct Rows {
  void* p = nullptr;
  int64_t sb = 0, sh = 0, st = 0;
  int hdiv = 1;
};

inline Rows rows_of(const dla_rows* r, int hdiv) {
  Rows x;
  if (r) {
    x.p = r->data;
    x.sb = r->stride_b;
    x.sh = r->stride_h;
    x.st = r->stride_t;
    x.hdiv = hdiv;
  }
  return x;
}

template <typename T>
__device__ __forceinline__ T* row_base(const Rows& r, int b, int h) {
  return static_cast<T*>(r.p) + (b * r.sb + (h / r.hdiv) * r.sh);
}

// What every kernel of a call is given.  Heads are numbered b * H + h.
struct RecArgs {
  int B, H, Hk, T, dk, dv;
  float scale;
  const int32_t* lengths;
  Rows gate;           // float32
  int nseg, seg_len;   // segments of seg_len tokens (a multiple of the chunk)
  float* seg_state;    // [heads][nseg][dk][dv], the state before each segment
  float* seg_adj;      // [heads][nseg][dk][dv], the adjoint behind each segment
  float* seg_decay;    // [heads][nseg]
  float2* decays;      // [heads][2][chunks * kRecChunk], see recurrence_tile.h
};

constexpr float kCutGate = -87.33655f;   // ln of 2^-126: a gate below it is a decay of zero
constexpr int kRecChunk = 32;   // tokens a workgroup takes at a time
__host__ __device__ inline int64_t rec_padded(int T) { return ((int64_t)T + kRecChunk - 1) / kRecChunk * kRecChunk; }

// Every token's decays within its chunk, for the chunk kernels of a call.
hipError_t launch_recurrence_decays(const RecArgs& a, hipStream_t st);

// Forward over segments: out (and the last state).
hipError_t launch_recurrence_forward(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                     const Rows& v, const Rows& out, const float* s0, float* s_out,
                                     hipStream_t st);
// dq, by the forward kernel with do, v, k in the places of q, k, v and the state
// transposed; qdot[head][t]: what the pairs (s < t, t) give to the gates between them;
// end_dot[head] = <dstate, last state> where dstate is given.
hipError_t launch_recurrence_dq(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                const Rows& v, const Rows& dout, const Rows& dq, bool dq_f32,
                                const float* s0, const float* dstate, float* qdot, float* end_dot,
                                hipStream_t st);
// dk, dv, dstate0 (ds0, which may be dstate's array), and kdot[head][t]: what the pairs (t,
// u > t) give to the gates between them.
hipError_t launch_recurrence_adjoint(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                     const Rows& v, const Rows& dout, const Rows& dk, bool dk_f32,
                                     const Rows& dv, const float* dstate, float* ds0, float* kdot,
                                     hipStream_t st);
// Each segment's own contribution to the state (or, reverse, to the adjoint), and from
// them the state before (the adjoint behind) each segment.  reverse, after the other: also
// anchor [heads][nseg][d_k d_v / 256], whose sums over the last axis are the products of the
// adjoint behind each segment but the last with the state there.
hipError_t launch_recurrence_segments(const RecArgs& a, int dtype, bool reverse, const Rows& x,
                                      const Rows& y, const float* first, double* anchor, hipStream_t st);
// Token by token, for short sequences.
hipError_t launch_recurrence_step(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                  const Rows& v, const Rows& out, const float* s0, float* s_out,
                                  hipStream_t st);
// dg from the per-token sums: dg_t = end_dot + sum over s >= t of (qdot_s - kdot_s), each
// segment's sum from its anchor.
hipError_t launch_recurrence_dgate(const RecArgs& a, int dtype, const float* qdot, const float* kdot,
                                   const double* anchor, const float* end_dot, const Rows& dg, hipStream_t st);
// Sums the heads that share a key head: [B][H][T][d] float32 -> rows of B * Hk heads.
hipError_t launch_head_sums(const RecArgs& a, int dtype, const float* dq_part, const Rows& dq,
                            const float* dk_part, const Rows& dk, hipStream_t st);

}  // namespace dla
