// The part of the recurrence's backward pass that runs from the last token back: dk, dv,
// the adjoint of the state, and the gate's gradient.
//
// With R the adjoint of the state behind a chunk (what later tokens and the last state's
// gradient ask of it), a chunk gives
//   dv_s = e^{a_end - a_s} R^T k_s + scale sum_{u >= s} e^{a_u - a_s} (q_u . k_s) do_u
//   dk_s = e^{a_end - a_s} R v_s   + scale sum_{u >= s} e^{a_u - a_s} (do_u . v_s) q_u
//   R   <- e^{a_end} R + scale sum_u e^{a_u} q_u do_u^T.
// dv contracts R over its rows and dk over its columns.  Half of the workgroup's waves hold
// 32 columns each of R, the others 32 columns each of R^T, in accumulators that are the
// operands of those products as they are; keeping R twice costs the products that update it
// and no pass through LDS.  Both halves run recurrence_tile.h's chunk step, back in time.
//
// The gate's gradient: e^{g_t} scales what every token s < t leaves for every token u >= t,
// so dg_t is the sum over those pairs of A_us = scale e^{a_u - a_s} (q_u . k_s)(do_u . v_s),
// with the state before all tokens and the gradient of the last one as further ends.  With
// x_u the sum of A_us over s < u and y_s that over u > s, dg_t = <dstate, last state> + sum
// over s >= t of (x_s - y_s).  No pair (t, t) enters either, so nothing large cancels where
// the gates are steep.  The dq pass leaves x (a lane holds a token u and its pairs' scores
// of do and v; each wave adds the products with its own 32 columns of q and k), this
// kernel y, the other way round.
#include "recurrence_tile.h"

namespace dla {
namespace {

// dg from the tokens' sums, from the last token back, in float64: what is added up spans
// the sequence, what is left may be small.  A cut gate lets nothing through: dg is zero
// there and the sum starts anew, exactly.  Two passes over blocks of tokens: each block's
// sum back to its first cut, then the tokens.
struct DgArgs {
  RecArgs a;
  const float* qdot;
  const float* kdot;
  const float* end_dot;
  double* block_sum;
  int* block_cut;
  Rows dg;
  int dtype;
};

constexpr int kPer = kDgateBlock / 256;

__device__ __forceinline__ void later(double& x, int& cut, double y, int ycut) {
  // x, cut: the part before; y, ycut: the part behind it
  if (!cut) x += y;
  cut |= ycut;
}

template <bool LAST>
__global__ __launch_bounds__(256) void dgate_kernel(DgArgs f) {
  const RecArgs& a = f.a;
  const int nb = gridDim.x, block = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const int b = head / a.H, h = head % a.H;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const float* gate = row_base<const float>(a.gate, b, h);
  __shared__ double sums[4];
  __shared__ int cuts[4];
  const int64_t t0 = (int64_t)block * kDgateBlock + tid * kPer;
  double x[kPer];
  int cut[kPer];
  double sum = 0.0;   // of the thread's tokens, from the last back to the first cut
  int any = 0;
#pragma unroll
  for (int i = kPer - 1; i >= 0; --i) {
    const int64_t t = t0 + i;
    x[i] = 0.0;
    cut[i] = 0;
    if (t < lim) {
      x[i] = (double)f.qdot[(int64_t)head * a.T + t] - (double)f.kdot[(int64_t)head * a.T + t];
      cut[i] = gate[t * a.gate.st] < kCutGate;
    }
    // a cut at t: what is at t and behind it counts for no earlier token
    double s = x[i];
    int c = cut[i];
    if (c) s = 0.0;
    later(s, c, sum, any);
    sum = s;
    any = c;
  }
  // this thread's sum and those of the threads behind it in the wave
  double ws = sum;
  int wc = any;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_down(ws, o);
    const int c = __shfl_down(wc, o);
    if (lane + o < 64) later(ws, wc, y, c);
  }
  if (lane == 0) {
    sums[wave] = ws;
    cuts[wave] = wc;
  }
  __syncthreads();
  if constexpr (!LAST) {
    if (tid == 0) {
      double s = sums[0];
      int c = cuts[0];
      for (int w = 1; w < 4; ++w) later(s, c, sums[w], cuts[w]);
      f.block_sum[(int64_t)head * nb + block] = s;
      f.block_cut[(int64_t)head * nb + block] = c;
    }
  } else {
    // what is behind this thread: the rest of its wave, the waves and blocks behind
    double s = __shfl_down(ws, 1);
    int c = __shfl_down(wc, 1);
    if (lane == 63) {
      s = 0.0;
      c = 0;
    }
    for (int w = wave + 1; w < 4; ++w) later(s, c, sums[w], cuts[w]);
    for (int i = block + 1; i < nb && !c; ++i)
      later(s, c, f.block_sum[(int64_t)head * nb + i], f.block_cut[(int64_t)head * nb + i]);
    if (!c && f.end_dot) s += (double)f.end_dot[head];
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
      const int64_t t = t0 + i;
      s = cut[i] ? 0.0 : s + x[i];
      if (t < a.T) {
        const float y = t < lim ? (float)s : 0.f;
        const int64_t at = b * f.dg.sb + h * f.dg.sh + t * f.dg.st;
        if (f.dtype == DLA_BF16) static_cast<__bf16*>(f.dg.p)[at] = (__bf16)y;
        else static_cast<float*>(f.dg.p)[at] = y;
      }
    }
  }
}

// [B][H][T][d] float32 -> the sum over the H / Hk heads of each key head, four columns a
// thread, heads in order.
template <typename Tin>
__global__ __launch_bounds__(256) void head_sum_kernel(RecArgs a, const float* part, Rows out) {
  const int n4 = a.dk / 4, G = a.H / a.Hk;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.T * n4;
  if (i >= per) return;
  const int64_t t = i / n4, c = 4 * (i % n4);
  const int b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk;
  const float* p = part + (((int64_t)b * a.H + hk * G) * a.T + t) * a.dk + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < G; ++j) {
    const float4 x = *reinterpret_cast<const float4*>(p + (int64_t)j * a.T * a.dk);
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
                                   const float* end_dot, double* block_sum, int* block_cut,
                                   const Rows& dg, hipStream_t st) {
  DgArgs f{a, qdot, kdot, end_dot, block_sum, block_cut, dg, dtype};
  const dim3 grid((a.T + kDgateBlock - 1) / kDgateBlock, a.B * a.H);
  if (grid.x > 1) hipLaunchKernelGGL((dgate_kernel<false>), grid, dim3(256), 0, st, f);
  hipLaunchKernelGGL((dgate_kernel<true>), grid, dim3(256), 0, st, f);
  return hipGetLastError();
}

hipError_t launch_head_sum(const RecArgs& a, int dtype, const float* part, const Rows& out,
                           hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.T * a.dk / 4 + 255) / 256), a.B * a.Hk);
  if (dtype == DLA_BF16) hipLaunchKernelGGL((head_sum_kernel<bf16_t>), grid, dim3(256), 0, st, a, part, out);
  else hipLaunchKernelGGL((head_sum_kernel<float>), grid, dim3(256), 0, st, a, part, out);
  return hipGetLastError();
}

}  // namespace dla
