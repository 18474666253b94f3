// The single-state recurrence over long sequences, and dq of its backward pass.
//
// A workgroup takes one head's segment of tokens, a chunk at a time (recurrence_tile.h
// has the chunk's formulas).  Wave w holds columns 32 w .. 32 w + 31 of the state, all
// d_k rows of them, in the accumulators of the products that update it; their layout is
// that of the first operand of the product that reads them, so the state never leaves
// the registers.  The chunk's scores are formed with keys as the first operand, which
// makes them, too, the operand of the product with the values; every wave forms them for
// itself, which costs a quarter more products and saves a barrier and a pass through LDS.
//
// dq_t = sum_{s <= t} e^{a_t - a_s} (do_t . v_s) k_s + e^{a_t} S do_t is the same with do,
// v and k in the places of q, k and v and the state transposed.  That pass also leaves
// qdot_t, what the pairs (s < t, t) give to the gates between them (recurrence_adjoint.hip).
#include "recurrence_tile.h"

namespace dla {
namespace {

struct FwdArgs {
  RecArgs a;
  Rows q, k, v, out;       // in the kernel's roles
  const float* s0;         // state before the first token, or null
  int64_t s_rs, s_cs;      // strides of a state's rows and columns, in the kernel's roles
  const float* seg_state;  // state before each segment, or null: one segment
  float* s_out;            // state behind the last token, or null
  const float* dstate;     // dq only, or null
  Rows x;                  // dq only: q
  float* qdot;
  float* end_dot;
  int out_f32;
};

// Decays of a chunk's tokens, a half-wave per chunk.
__global__ __launch_bounds__(256) void decays_kernel(RecArgs a) {
  const int64_t padded = rec_padded(a.T), chunks = padded / kChunk;
  const int lane = threadIdx.x & 31;
  const int64_t c = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int head = blockIdx.y, b = head / a.H, h = head % a.H;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int64_t t = c * kChunk + lane;
  const float gate = t < lim ? row_base<const float>(a.gate, b, h)[t * a.gate.st] : 0.f;
  const bool cut = gate < kCutGate;
  double x = cut ? 0.0 : (double)gate * 1.4426950408889634;
  int n = cut ? 1 : 0;
#pragma unroll
  for (int o = 1; o < kChunk; o <<= 1) {
    const double y = __shfl_up(x, o, kChunk);
    const int m = __shfl_up(n, o, kChunk);
    if (lane >= o) {
      x += y;
      n += m;
    }
  }
  const double w = rint(x);
  const float hi = (float)w - 131072.f * (float)n, lo = (float)(x - w);
  const float eh = __shfl(hi, kChunk - 1, kChunk), el = __shfl(lo, kChunk - 1, kChunk);
  if (c < chunks)
    a.decays[head * padded + t] = make_float4(hi, lo, decay2(hi, lo, 0.f, 0.f), decay2(eh, el, hi, lo));
}

// A chunk's tiles; two of them, so that the next chunk is stored while one is read and a
// chunk takes one barrier.
template <typename Tin, int DK, int DV, bool DQ>
struct FwdTiles {
  Tin q[kChunk * DK], k[kChunk * DK], v[kChunk * DV], x[DQ ? kChunk * DV : 8];
  Decays dec;
  float dots[DQ ? DV / 32 : 1][kChunk];
};

template <typename Tin, int DK, int DV, bool DQ>
__global__ __launch_bounds__(2 * DV, sizeof(Tin) == 2 ? 2 : 1) void forward_kernel(FwdArgs f) {
  constexpr int NT = 2 * DV, NW = DV / 32, ST = DK / 32;
  __shared__ __align__(16) FwdTiles<Tin, DK, DV, DQ> tiles[2];
  const RecArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5;
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H, c0 = 32 * wave;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const Tin* q = row_base<const Tin>(f.q, b, h);
  const Tin* k = row_base<const Tin>(f.k, b, h);
  const Tin* v = row_base<const Tin>(f.v, b, h);
  const Tin* x = DQ ? row_base<const Tin>(f.x, b, h) : nullptr;
  const float4* decays = a.decays + head * rec_padded(a.T);
  const int64_t D = (int64_t)DK * DV;

  Stage<Tin, DK, NT> gq, gk;
  Stage<Tin, DV, NT> gv, gx;
  float4 gd;
  auto request = [&](int t0) {
    gq.load(q, f.q.st, t0, lim, tid);
    gk.load(k, f.k.st, t0, lim, tid);
    gv.load(v, f.v.st, t0, lim, tid);
    if constexpr (DQ) gx.load(x, f.x.st, t0, lim, tid);
    if (tid < kChunk) gd = decays[t0 + tid];
  };
  auto store = [&](FwdTiles<Tin, DK, DV, DQ>& to) {
    gq.store(to.q, tid);
    gk.store(to.k, tid);
    gv.store(to.v, tid);
    if constexpr (DQ) gx.store(to.x, tid);
    if (tid < kChunk) to.dec.store(gd, tid);
  };
  request(begin);
  f32x16 S[ST];
  const float* first = f.seg_state ? f.seg_state + ((int64_t)head * a.nseg + seg) * D
                                   : (f.s0 ? f.s0 + head * D : nullptr);
  if (first) {
    load_state(S, first, f.s_rs, f.s_cs, c0, lane);
  } else {
#pragma unroll
    for (int i = 0; i < ST; ++i) S[i] = zero16();
  }
  store(tiles[0]);
  __syncthreads();
  int at = 0;
  // the waves' parts of a chunk's dots, added up by the chunk's successor
  auto sum_dots = [&](const FwdTiles<Tin, DK, DV, DQ>& from, int t0) {
    if (tid < kChunk && t0 + tid < end) {
      float y = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) y += from.dots[w][tid];
      f.qdot[(int64_t)head * a.T + t0 + tid] = t0 + tid < lim ? y : 0.f;
    }
  };
  for (int t0 = begin; t0 < end; t0 += kChunk, at ^= 1) {
    FwdTiles<Tin, DK, DV, DQ>& now = tiles[at];
    if constexpr (DQ) {
      if (t0 > begin) sum_dots(tiles[at ^ 1], t0 - kChunk);
    }
    if (t0 + kChunk < end) request(t0 + kChunk);
    const int t = t0 + (lane & 31);
    f32x16 o;
    const float dot = chunk_step<Tin, DK, DV, false, DQ>(now.q, now.k, now.v, now.x, now.dec, a.scale, c0, lane, S, o);
    if constexpr (DQ) {
      if (g == 0) now.dots[wave][lane] = dot;
    }
    if (t >= lim) o = zero16();
    if (t < end) {
      if (DQ && f.out_f32) store_out(row_base<float>(f.out, b, h) + t * f.out.st, c0, o, lane);
      else store_out(row_base<Tin>(f.out, b, h) + t * f.out.st, c0, o, lane);
    }
    if (t0 + kChunk < end) store(tiles[at ^ 1]);
    __syncthreads();
  }
  if constexpr (DQ) sum_dots(tiles[at ^ 1], begin + (end - begin - 1) / kChunk * kChunk);
  if (seg == a.nseg - 1) {
    if (f.s_out) store_state(S, f.s_out + head * D, f.s_rs, f.s_cs, c0, lane);
    if constexpr (DQ) {
      if (f.dstate) {
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            y += S[i][r] * f.dstate[head * D + (32 * i + held_row(r, lane)) * f.s_rs +
                                    (c0 + perm_row(lane & 31)) * f.s_cs];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) y += __shfl_xor(y, o);
        if (lane == 0) tiles[at].dots[wave][0] = y;
        __syncthreads();
        if (tid == 0) {
          float z = 0.f;
          for (int w = 0; w < NW; ++w) z += tiles[at].dots[w][0];
          f.end_dot[head] = z;
        }
      }
    }
  }
}

// A segment's own part of the state behind it, sum over its tokens of (decay to the
// segment's end) k_s v_s^T; reverse: of the adjoint before it, sum of scale (decay from
// the segment's start) q_s do_s^T.
template <typename Tin, int DK, int DV>
struct SegTiles {
  Tin k[kChunk * DK], v[kChunk * DV];
  Decays dec;
};

template <typename Tin, int DK, int DV, bool REV>
__global__ __launch_bounds__(2 * DV, sizeof(Tin) == 2 ? 2 : 1) void segment_kernel(RecArgs a, Rows xr, Rows yr, float* dst) {
  constexpr int NT = 2 * DV, ST = DK / 32;
  __shared__ __align__(16) SegTiles<Tin, DK, DV> tiles[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H, c0 = 32 * wave;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const Tin* x = row_base<const Tin>(xr, b, h);
  const Tin* y = row_base<const Tin>(yr, b, h);
  const float4* decays = a.decays + head * rec_padded(a.T);
  f32x16 S[ST];
#pragma unroll
  for (int i = 0; i < ST; ++i) S[i] = zero16();
  float decay = 1.f;
  Stage<Tin, DK, NT> gx;
  Stage<Tin, DV, NT> gy;
  float4 gd;
  auto request = [&](int t0) {
    gx.load(x, xr.st, t0, lim, tid);
    gy.load(y, yr.st, t0, lim, tid);
    if (tid < kChunk) gd = decays[t0 + tid];
  };
  auto store = [&](SegTiles<Tin, DK, DV>& to) {
    gx.store(to.k, tid);
    gy.store(to.v, tid);
    if (tid < kChunk) to.dec.store(gd, tid);
  };
  const int n = (end - begin + kChunk - 1) / kChunk;
  auto chunk_at = [&](int c) { return begin + (REV ? n - 1 - c : c) * kChunk; };
  request(chunk_at(0));
  store(tiles[0]);
  __syncthreads();
  for (int c = 0; c < n; ++c) {
    const SegTiles<Tin, DK, DV>& now = tiles[c & 1];
    if (c + 1 < n) request(chunk_at(c + 1));
    const float total = now.dec.total();
    decay *= total;
#pragma unroll
    for (int i = 0; i < ST; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[i][r] *= total;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      float w[8];
      weights8(REV ? now.dec.in : now.dec.out, kk, lane, w);
      if constexpr (REV) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] *= a.scale;
      }
      const Scaled<Tin> z(Tile<Tin, DV>::col_frag(now.v, c0, kk, lane), w);
#pragma unroll
      for (int i = 0; i < ST; ++i) z.mma_b(S[i], Tile<Tin, DK>::col_frag(now.k, 32 * i, kk, lane));
    }
    if (c + 1 < n) store(tiles[(c + 1) & 1]);
    __syncthreads();
  }
  store_state(S, dst + ((int64_t)head * a.nseg + seg) * DK * DV, DV, 1, c0, lane);
  if (tid == 0) a.seg_decay[(int64_t)head * a.nseg + seg] = decay;
}

// The segments' own parts become the states before them (reverse: the adjoints behind
// them), one element of a head's state per thread.
template <bool REV>
__global__ __launch_bounds__(256) void prefix_kernel(RecArgs a, float* part, const float* first) {
  const int64_t D = (int64_t)a.dk * a.dv;
  const int head = blockIdx.y;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;   // D is a multiple of 256
  float* p = part + (int64_t)head * a.nseg * D + i;
  const float* decay = a.seg_decay + (int64_t)head * a.nseg;
  float cur = first ? first[head * D + i] : 0.f;
  for (int j = 0; j < a.nseg; ++j) {
    const int s = REV ? a.nseg - 1 - j : j;
    const float own = p[s * D];
    p[s * D] = cur;
    cur = decay[s] * cur + own;
  }
}

template <typename Tin, int DK, int DV, bool DQ>
hipError_t run_forward(const FwdArgs& f, hipStream_t st) {
  const int grid = f.a.B * f.a.H * f.a.nseg;
  hipLaunchKernelGGL((forward_kernel<Tin, DK, DV, DQ>), dim3(grid), dim3(2 * DV), 0, st, f);
  return hipGetLastError();
}

template <bool DQ>
hipError_t pick_forward(const FwdArgs& f, int dtype, int dk, int dv, hipStream_t st) {
  if (dtype == DLA_BF16) {
    if (dk == 128) return dv == 128 ? run_forward<bf16_t, 128, 128, DQ>(f, st) : run_forward<bf16_t, 128, 64, DQ>(f, st);
    return dv == 128 ? run_forward<bf16_t, 64, 128, DQ>(f, st) : run_forward<bf16_t, 64, 64, DQ>(f, st);
  }
  if (dk == 128) return dv == 128 ? run_forward<float, 128, 128, DQ>(f, st) : run_forward<float, 128, 64, DQ>(f, st);
  return dv == 128 ? run_forward<float, 64, 128, DQ>(f, st) : run_forward<float, 64, 64, DQ>(f, st);
}

template <typename Tin, int DK, int DV>
hipError_t run_segments(const RecArgs& a, bool rev, const Rows& x, const Rows& y, const float* first,
                        hipStream_t st) {
  const dim3 grid(a.B * a.H * a.nseg), block(2 * DV), pg(DK * DV / 256, a.B * a.H);
  float* dst = rev ? a.seg_adj : a.seg_state;
  if (rev) {
    hipLaunchKernelGGL((segment_kernel<Tin, DK, DV, true>), grid, block, 0, st, a, x, y, dst);
    hipLaunchKernelGGL((prefix_kernel<true>), pg, dim3(256), 0, st, a, dst, first);
  } else {
    hipLaunchKernelGGL((segment_kernel<Tin, DK, DV, false>), grid, block, 0, st, a, x, y, dst);
    hipLaunchKernelGGL((prefix_kernel<false>), pg, dim3(256), 0, st, a, dst, first);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_recurrence_decays(const RecArgs& a, hipStream_t st) {
  const int64_t chunks = rec_padded(a.T) / kChunk;
  hipLaunchKernelGGL(decays_kernel, dim3((unsigned)((chunks + 7) / 8), a.B * a.H), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_recurrence_segments(const RecArgs& a, int dtype, bool reverse, const Rows& x,
                                      const Rows& y, const float* first, hipStream_t st) {
  if (dtype == DLA_BF16) {
    if (a.dk == 128) return a.dv == 128 ? run_segments<bf16_t, 128, 128>(a, reverse, x, y, first, st) : run_segments<bf16_t, 128, 64>(a, reverse, x, y, first, st);
    return a.dv == 128 ? run_segments<bf16_t, 64, 128>(a, reverse, x, y, first, st) : run_segments<bf16_t, 64, 64>(a, reverse, x, y, first, st);
  }
  if (a.dk == 128) return a.dv == 128 ? run_segments<float, 128, 128>(a, reverse, x, y, first, st) : run_segments<float, 128, 64>(a, reverse, x, y, first, st);
  return a.dv == 128 ? run_segments<float, 64, 128>(a, reverse, x, y, first, st) : run_segments<float, 64, 64>(a, reverse, x, y, first, st);
}

hipError_t launch_recurrence_forward(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                     const Rows& v, const Rows& out, const float* s0, float* s_out,
                                     hipStream_t st) {
  FwdArgs f;
  f.a = a;
  f.q = q;
  f.k = k;
  f.v = v;
  f.out = out;
  f.s0 = s0;
  f.s_rs = a.dv;
  f.s_cs = 1;
  f.seg_state = a.nseg > 1 ? a.seg_state : nullptr;
  f.s_out = s_out;
  f.dstate = nullptr;
  f.qdot = f.end_dot = nullptr;
  f.out_f32 = 0;
  return pick_forward<false>(f, dtype, a.dk, a.dv, st);
}

hipError_t launch_recurrence_dq(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                const Rows& v, const Rows& dout, const Rows& dq, bool dq_f32,
                                const float* s0, const float* dstate, float* qdot, float* end_dot,
                                hipStream_t st) {
  FwdArgs f;
  f.a = a;
  f.q = dout;
  f.k = v;
  f.v = k;
  f.out = dq;
  f.s0 = s0;
  f.s_rs = 1;
  f.s_cs = a.dv;
  f.seg_state = a.nseg > 1 ? a.seg_state : nullptr;
  f.s_out = nullptr;
  f.dstate = dstate;
  f.x = q;
  f.qdot = qdot;
  f.end_dot = end_dot;
  f.out_f32 = dq_f32 ? 1 : 0;
  return pick_forward<true>(f, dtype, a.dv, a.dk, st);
}

}  // namespace dla
