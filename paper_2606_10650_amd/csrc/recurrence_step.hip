// The single-state recurrence token by token, for the few tokens of a decode step.
//
// A workgroup takes 32 columns of one head's state: they are independent of the others.
// Thread r 8 + c holds rows r, r + 32, .. of columns 4 c .. 4 c + 3 in registers, read and
// written once for all tokens of the call; the state's bytes bound it: 2048 heads of 128 x 128
// 41 us for 0.27 GB a token where calls follow on one state, part of which stays in the last
// cache; 32 heads 4.3, a launch.
#include "mfma.h"
#include "recurrence.h"

namespace dla {
namespace {

template <typename Tin, int DK>
__global__ __launch_bounds__(256) void step_kernel(RecArgs a, Rows q, Rows k, Rows v, Rows out,
                                                   const float* s0, float* s_out) {
  constexpr int NR = DK / 32;
  __shared__ float4 part[4][8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cb = a.dv / 32, head = blockIdx.x / cb, b = head / a.H, h = head % a.H;
  const int col = 32 * (blockIdx.x % cb) + 4 * (tid & 7), row = tid >> 3;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int64_t at = (int64_t)head * DK * a.dv + (int64_t)row * a.dv + col;
  float4 S[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i)
    S[i] = s0 ? *reinterpret_cast<const float4*>(s0 + at + (int64_t)32 * i * a.dv)
              : make_float4(0.f, 0.f, 0.f, 0.f);
  const Tin* qp = row_base<const Tin>(q, b, h) + row;
  const Tin* kp = row_base<const Tin>(k, b, h) + row;
  const Tin* vp = row_base<const Tin>(v, b, h) + col;
  const float* gate = row_base<const float>(a.gate, b, h);
  for (int t = 0; t < a.T; ++t) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t < lim) {
      const float x = gate[t * a.gate.st], d = x < kCutGate ? 0.f : expf(x);
      float y[4];
      load4f(vp + t * v.st, y);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float kk = to_f32(kp[t * k.st + 32 * i]), qq = to_f32(qp[t * q.st + 32 * i]);
        S[i].x = d * S[i].x + kk * y[0];
        S[i].y = d * S[i].y + kk * y[1];
        S[i].z = d * S[i].z + kk * y[2];
        S[i].w = d * S[i].w + kk * y[3];
        o.x += qq * S[i].x;
        o.y += qq * S[i].y;
        o.z += qq * S[i].z;
        o.w += qq * S[i].w;
      }
    }
#pragma unroll
    for (int m = 8; m < 64; m <<= 1) {
      o.x += __shfl_xor(o.x, m);
      o.y += __shfl_xor(o.y, m);
      o.z += __shfl_xor(o.z, m);
      o.w += __shfl_xor(o.w, m);
    }
    if (t > 0) __syncthreads();
    if (lane < 8) part[wave][lane] = o;
    __syncthreads();
    if (tid < 8) {
      const float4 p0 = part[0][tid], p1 = part[1][tid], p2 = part[2][tid], p3 = part[3][tid];
      Tin* r = row_base<Tin>(out, b, h) + t * out.st + col;
      const float c = a.scale;
      const float x[4] = {c * ((p0.x + p1.x) + (p2.x + p3.x)), c * ((p0.y + p1.y) + (p2.y + p3.y)),
                          c * ((p0.z + p1.z) + (p2.z + p3.z)), c * ((p0.w + p1.w) + (p2.w + p3.w))};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(Tin) == 2) reinterpret_cast<__bf16*>(r)[j] = (__bf16)x[j];
        else r[j] = x[j];
      }
    }
  }
  if (s_out) {
#pragma unroll
    for (int i = 0; i < NR; ++i)
      *reinterpret_cast<float4*>(s_out + at + (int64_t)32 * i * a.dv) = S[i];
  }
}

}  // namespace

hipError_t launch_recurrence_step(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                  const Rows& v, const Rows& out, const float* s0, float* s_out,
                                  hipStream_t st) {
  const dim3 grid(a.B * a.H * (a.dv / 32));
  if (dtype == DLA_BF16) {
    if (a.dk == 128) hipLaunchKernelGGL((step_kernel<bf16_t, 128>), grid, dim3(256), 0, st, a, q, k, v, out, s0, s_out);
    else hipLaunchKernelGGL((step_kernel<bf16_t, 64>), grid, dim3(256), 0, st, a, q, k, v, out, s0, s_out);
  } else {
    if (a.dk == 128) hipLaunchKernelGGL((step_kernel<float, 128>), grid, dim3(256), 0, st, a, q, k, v, out, s0, s_out);
    else hipLaunchKernelGGL((step_kernel<float, 64>), grid, dim3(256), 0, st, a, q, k, v, out, s0, s_out);
  }
  return hipGetLastError();
}

}  // namespace dla
