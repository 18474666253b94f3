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

struct AdjArgs {
  RecArgs a;
  Rows q, k, v, dout, dk, dv;
  const float* dstate;
  float* ds0;
  float* kdot;   // [heads][T]: y_s
  int dk_f32;
};

template <typename Tin, int DK, int DV>
struct AdjTiles {
  Tin q[kChunk * DK], k[kChunk * DK], v[kChunk * DV], o[kChunk * DV];
  Decays dec;
  float dots[DK / 32][kChunk];
};

// Waves 0 .. DV / 32 - 1 hold 32 columns each of R [DK][DV] and give dv; the others hold
// those of its transpose and give dk.
template <typename Tin, int DK, int DV>
__global__ __launch_bounds__(2 * (DK + DV), 1) void adjoint_kernel(AdjArgs f) {
  constexpr int NT = 2 * (DK + DV), KW = DK / 32, VW = DV / 32;
  using Tiles = AdjTiles<Tin, DK, DV>;
  __shared__ __align__(16) Tiles tiles[2];
  const RecArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5;
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H;
  const bool of_v = wave < VW;
  const int kw = wave - VW, c0 = 32 * (of_v ? wave : kw);
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const Tin* q = row_base<const Tin>(f.q, b, h);
  const Tin* k = row_base<const Tin>(f.k, b, h);
  const Tin* v = row_base<const Tin>(f.v, b, h);
  const Tin* dout = row_base<const Tin>(f.dout, b, h);
  const float4* decays = a.decays + head * rec_padded(a.T);
  const int64_t D = (int64_t)DK * DV;

  Stage<Tin, DK, NT> gq, gk;
  Stage<Tin, DV, NT> gv, go;
  float4 gd;
  auto request = [&](int t0) {
    gq.load(q, f.q.st, t0, lim, tid);
    gk.load(k, f.k.st, t0, lim, tid);
    gv.load(v, f.v.st, t0, lim, tid);
    go.load(dout, f.dout.st, t0, lim, tid);
    if (tid < kChunk) gd = decays[t0 + tid];
  };
  auto store = [&](Tiles& to) {
    gq.store(to.q, tid);
    gk.store(to.k, tid);
    gv.store(to.v, tid);
    go.store(to.o, tid);
    if (tid < kChunk) to.dec.store(gd, tid);
  };
  const float* last = a.nseg > 1 ? a.seg_adj + ((int64_t)head * a.nseg + seg) * D
                                 : (f.dstate ? f.dstate + head * D : nullptr);
  const int t_last = begin + (end - begin - 1) / kChunk * kChunk;
  request(t_last);
  int at = 0;
  if (of_v) {
    f32x16 R[DK / 32];
#pragma unroll
    for (int i = 0; i < DK / 32; ++i) R[i] = zero16();
    if (last) load_state(R, last, DV, 1, c0, lane);
    store(tiles[0]);
    __syncthreads();
    for (int t0 = t_last; t0 >= begin; t0 -= kChunk, at ^= 1) {
      const Tiles& now = tiles[at];
      if (t0 > begin) request(t0 - kChunk);
      const int s = t0 + (lane & 31);
      f32x16 o;
      chunk_step<Tin, DK, DV, true, false>(now.k, now.q, now.o, nullptr, now.dec, a.scale, c0, lane, R, o);
      if (s >= lim) o = zero16();
      if (s < end) store_out(row_base<Tin>(f.dv, b, h) + s * f.dv.st, c0, o, lane);
      if (t0 > begin) store(tiles[at ^ 1]);
      __syncthreads();
    }
    if (seg == 0 && f.ds0) store_state(R, f.ds0 + head * D, DV, 1, c0, lane);
  } else {
    f32x16 R[DV / 32];
#pragma unroll
    for (int i = 0; i < DV / 32; ++i) R[i] = zero16();
    if (last) load_state(R, last, 1, DV, c0, lane);
    // the waves' parts of a chunk's dots, added up by the chunk's successor
    auto sum_dots = [&](const Tiles& from, int t0) {
      if (kw == 0 && lane < kChunk && t0 + lane < end) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < KW; ++i) x += from.dots[i][lane];
        f.kdot[(int64_t)head * a.T + t0 + lane] = t0 + lane < lim ? x : 0.f;
      }
    };
    store(tiles[0]);
    __syncthreads();
    for (int t0 = t_last; t0 >= begin; t0 -= kChunk, at ^= 1) {
      Tiles& now = tiles[at];
      if (t0 < t_last) sum_dots(tiles[at ^ 1], t0 + kChunk);
      if (t0 > begin) request(t0 - kChunk);
      const int s = t0 + (lane & 31);
      f32x16 o;
      const float dot = chunk_step<Tin, DV, DK, true, true>(now.v, now.o, now.q, now.k, now.dec, a.scale, c0, lane, R, o);
      if (g == 0) now.dots[kw][lane] = dot;
      if (s >= lim) o = zero16();
      if (s < end) {
        if (f.dk_f32) store_out(row_base<float>(f.dk, b, h) + s * f.dk.st, c0, o, lane);
        else store_out(row_base<Tin>(f.dk, b, h) + s * f.dk.st, c0, o, lane);
      }
      if (t0 > begin) store(tiles[at ^ 1]);
      __syncthreads();
    }
    sum_dots(tiles[at ^ 1], begin);
  }
}

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

template <typename Tin, int DK, int DV>
hipError_t run_adjoint(const AdjArgs& f, hipStream_t st) {
  hipLaunchKernelGGL((adjoint_kernel<Tin, DK, DV>), dim3(f.a.B * f.a.H * f.a.nseg),
                     dim3(2 * (DK + DV)), 0, st, f);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_recurrence_adjoint(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                     const Rows& v, const Rows& dout, const Rows& dk, bool dk_f32,
                                     const Rows& dv, const float* dstate, float* ds0, float* kdot,
                                     hipStream_t st) {
  AdjArgs f;
  f.a = a;
  f.q = q;
  f.k = k;
  f.v = v;
  f.dout = dout;
  f.dk = dk;
  f.dv = dv;
  f.dstate = dstate;
  f.ds0 = ds0;
  f.kdot = kdot;
  f.dk_f32 = dk_f32 ? 1 : 0;
  if (dtype == DLA_BF16) {
    if (a.dk == 128) return a.dv == 128 ? run_adjoint<bf16_t, 128, 128>(f, st) : run_adjoint<bf16_t, 128, 64>(f, st);
    return a.dv == 128 ? run_adjoint<bf16_t, 64, 128>(f, st) : run_adjoint<bf16_t, 64, 64>(f, st);
  }
  if (a.dk == 128) return a.dv == 128 ? run_adjoint<float, 128, 128>(f, st) : run_adjoint<float, 128, 64>(f, st);
  return a.dv == 128 ? run_adjoint<float, 64, 128>(f, st) : run_adjoint<float, 64, 64>(f, st);
}

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
