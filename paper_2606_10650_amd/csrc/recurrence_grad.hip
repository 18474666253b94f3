// What the recurrence's backward pass adds up: the gate's gradient, and dq and dk over heads
// that share keys.
//
// The gate's gradient: e^{g_t} scales what every token s < t leaves for every token u >= t,
// so dg_t is the sum over those pairs of A_us = scale e^{a_u - a_s} (q_u . k_s)(do_u . v_s),
// with the state before all tokens and the gradient of the last one as further ends.  With
// x_u the sum of A_us over s < u and y_s that over u > s, dg_t = <dstate, last state> + sum
// over s >= t of (x_s - y_s).  No pair (t, t) enters either, so nothing large cancels where
// the gates are steep.  dg is rounded once, to the inputs' type: gates are a projection of the
// same type, whose backward pass multiplies their gradient in that type.  The dq pass leaves x (a lane holds a token u and its pairs' scores
// of do and v; each wave adds the products with its own 32 columns of q and k), the dk pass
// y, the other way round.
#include "recurrence_tile.h"

namespace dla {
namespace {

// dg from the tokens' sums, from the last token back, in float64: what is added up spans
// many tokens, what is left may be small.  Each segment starts from its own end, where the
// sum is <adjoint behind the segment, state there> (parts of 256 elements, prefix_kernel), so
// that what the tokens' sums were rounded by adds up over a segment at most.  A cut gate lets
// nothing through: dg is zero there and the sum starts anew, exactly.
struct DgArgs {
  RecArgs a;
  const float* qdot;
  const float* kdot;
  const double* anchor;   // [heads][nseg][d_k d_v / 256], the last segment's apart:
  const float* end_dot;   // [heads], or null for zero
  Rows dg;
  int dtype;
};

constexpr int kPer = 4, kDgateBlock = 256 * kPer;

// x, cut: the sum of a run of tokens back to its first cut, and whether it has one; takes
// the run behind it
__device__ __forceinline__ void later(double& x, int& cut, double y, int ycut) {
  if (!cut) x += y;
  cut |= ycut;
}

__global__ __launch_bounds__(256) void dgate_kernel(DgArgs f) {
  const RecArgs& a = f.a;
  const int seg = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = head / a.H, h = head % a.H;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const float* gate = row_base<const float>(a.gate, b, h);
  const float* qd = f.qdot + (int64_t)head * a.T;
  const float* kd = f.kdot + (int64_t)head * a.T;
  __shared__ double sums[4];
  __shared__ int cuts[4];
  double carry = 0.0;   // of what is behind the block
  if (seg < a.nseg - 1) {
    const int n = a.dk * a.dv / 256;   // up to 64: every wave adds them up
    if (lane < n) carry = f.anchor[((int64_t)head * a.nseg + seg) * n + lane];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) carry += __shfl_xor(carry, o);
  } else if (f.end_dot) carry = (double)f.end_dot[head];
  for (int base = begin + (end - begin - 1) / kDgateBlock * kDgateBlock; base >= begin; base -= kDgateBlock) {
    const int t0 = base + tid * kPer;
    double x[kPer];
    int cut[kPer];
    double sum = 0.0;   // of the thread's tokens, from the last back to the first cut
    int any = 0;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
      const int t = t0 + i;
      x[i] = 0.0;
      cut[i] = 0;
      if (t < end && t < lim) {
        x[i] = (double)qd[t] - (double)kd[t];
        cut[i] = gate[t * a.gate.st] < kCutGate;
      }
      // a cut at t: it and what is behind it count for no earlier token
      sum = cut[i] ? 0.0 : sum + x[i];
      any |= cut[i];
    }
    double ws = sum;   // with the threads behind it in the wave
    int wc = any;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_down(ws, o);
      const int c = __shfl_down(wc, o);
      if (lane + o < 64) later(ws, wc, y, c);
    }
    __syncthreads();   // the last block's sums are read
    if (lane == 0) {
      sums[wave] = ws;
      cuts[wave] = wc;
    }
    __syncthreads();
    // what is behind this thread: the rest of its wave, the waves behind, the blocks behind
    double s = __shfl_down(ws, 1);
    int c = __shfl_down(wc, 1);
    if (lane == 63) {
      s = 0.0;
      c = 0;
    }
    for (int w = wave + 1; w < 4; ++w) later(s, c, sums[w], cuts[w]);
    later(s, c, carry, 0);
    double all = sums[0];
    c = cuts[0];
    for (int w = 1; w < 4; ++w) later(all, c, sums[w], cuts[w]);
    later(all, c, carry, 0);
    carry = all;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
      const int t = t0 + i;
      s = cut[i] ? 0.0 : s + x[i];
      if (t < end) {
        const float y = t < lim ? (float)s : 0.f;
        const int64_t at = b * f.dg.sb + h * f.dg.sh + t * f.dg.st;
        if (f.dtype == DLA_BF16) static_cast<__bf16*>(f.dg.p)[at] = (__bf16)y;
        else static_cast<float*>(f.dg.p)[at] = y;
      }
    }
  }
}

// [B][H][T][d] float32 -> the sum over the H / Hk heads of each key head, four columns a
// thread, heads in order, of dq and of dk in one launch.
struct HeadSums {
  const float* part[2];
  Rows out[2];
};

template <typename Tin>
__global__ __launch_bounds__(256) void head_sum_kernel(RecArgs a, HeadSums f) {
  const int n4 = a.dk / 4, G = a.H / a.Hk;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.T * n4;
  if (i >= per) return;
  const int64_t t = i / n4, c = 4 * (i % n4), step = (int64_t)a.T * a.dk;
  const int b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk;
  const Rows& out = f.out[blockIdx.z];
  const float* p = f.part[blockIdx.z] + (((int64_t)b * a.H + hk * G) * a.T + t) * a.dk + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int j = 0; j < G; ++j) {
    const float4 x = *reinterpret_cast<const float4*>(p + j * step);
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  Tin* dst = static_cast<Tin*>(out.p) + b * out.sb + hk * out.sh + t * out.st + c;
  if constexpr (sizeof(Tin) == 2) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 y;
    y[0] = (__bf16)s.x;
    y[1] = (__bf16)s.y;
    y[2] = (__bf16)s.z;
    y[3] = (__bf16)s.w;
    *reinterpret_cast<bf16x4*>(dst) = y;
  } else {
    *reinterpret_cast<float4*>(dst) = s;
  }
}

}  // namespace

hipError_t launch_recurrence_dgate(const RecArgs& a, int dtype, const float* qdot, const float* kdot,
                                   const double* anchor, const float* end_dot, const Rows& dg, hipStream_t st) {
  const DgArgs f{a, qdot, kdot, anchor, end_dot, dg, dtype};
  hipLaunchKernelGGL(dgate_kernel, dim3(a.nseg, a.B * a.H), dim3(256), 0, st, f);
  return hipGetLastError();
}

hipError_t launch_head_sums(const RecArgs& a, int dtype, const float* dq_part, const Rows& dq,
                            const float* dk_part, const Rows& dk, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.T * a.dk / 4 + 255) / 256), a.B * a.Hk, 2);
  const HeadSums f{{dq_part, dk_part}, {dq, dk}};
  if (dtype == DLA_BF16) hipLaunchKernelGGL((head_sum_kernel<bf16_t>), grid, dim3(256), 0, st, a, f);
  else hipLaunchKernelGGL((head_sum_kernel<float>), grid, dim3(256), 0, st, a, f);
  return hipGetLastError();
}

}  // namespace dla
