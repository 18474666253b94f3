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
// qdot_t, what the pairs (s < t, t) give to the gates between them (recurrence_grad.hip).
#include "recurrence_tile.h"

namespace dla {
namespace {

// One pass over the tokens, in the kernel's roles: q, k of R values and v of C, a state
// [R][C], out of C.
struct ScanArgs {
  RecArgs a;
  Rows q, k, v, out;
  Rows y;                  // PAIR: rows of C whose products with the pass's output go to dot
  const float* first;      // the state before the pass's first token, per head, or null
  int64_t s_rs, s_cs;      // strides of a state's rows and columns
  const float* seg_first;  // the state before each segment, or null: one segment
  float* last;             // the state behind the pass's last token, or null
  float* dot;              // PAIR: [heads][T]
  const float* end_with;   // PAIR: per head, or null; end_dot = <end_with, last state>
  float* end_dot;
  int out_f32;             // PAIR: out is float32
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
  if (c < chunks) {
    float2* d = a.decays + 2 * head * padded;
    d[t] = make_float2(hi, lo);
    d[padded + t] = make_float2(decay2(hi, lo, 0.f, 0.f), decay2(eh, el, hi, lo));
  }
}

template <typename Tin, int R, int C, bool PAIR>
struct ScanTiles {
  Tin q[Tile<Tin, R>::SIZE], k[Tile<Tin, R>::SIZE], v[Tile<Tin, C>::SIZE], y[PAIR ? Tile<Tin, C>::SIZE : 8];
  Decays dec;
  float dots[PAIR ? C / 32 : 1][kChunk];
};

// REV: from the segment's last chunk to its first.
template <typename Tin, int R, int C, bool REV, bool PAIR>
__global__ __launch_bounds__(2 * C, sizeof(Tin) == 2 ? 2 : 1) void scan_kernel(ScanArgs f) {
  constexpr int NT = 2 * C, NW = C / 32;
  __shared__ __align__(16) ScanTiles<Tin, R, C, PAIR> now;
  const RecArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H, c0 = 32 * wave;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const Tin* q = row_base<const Tin>(f.q, b, h);
  const Tin* k = row_base<const Tin>(f.k, b, h);
  const Tin* v = row_base<const Tin>(f.v, b, h);
  const Tin* y = PAIR ? row_base<const Tin>(f.y, b, h) : nullptr;
  const int64_t D = (int64_t)R * C, padded = rec_padded(a.T);
  const float2* decays = a.decays + 2 * head * padded;

  Stage<Tin, R, NT> gq, gk;
  Stage<Tin, C, NT> gv, gy;
  DecayStage<NT, REV> gd;
  auto request = [&](int t0) {
    gq.load(q + t0 * f.q.st, f.q.st, lim - t0, tid);
    gk.load(k + t0 * f.k.st, f.k.st, lim - t0, tid);
    gv.load(v + t0 * f.v.st, f.v.st, lim - t0, tid);
    if constexpr (PAIR) gy.load(y + t0 * f.y.st, f.y.st, lim - t0, tid);
    gd.load(decays, padded, t0, tid);
  };
  // the waves' parts of a chunk's dots, added up when the next one's tokens are staged
  auto sum_dots = [&](int t0) {
    if (tid < kChunk && t0 + tid < end) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) x += now.dots[w][tid];
      f.dot[(int64_t)head * a.T + t0 + tid] = t0 + tid < lim ? x : 0.f;
    }
  };
  const int n = (end - begin + kChunk - 1) / kChunk;
  auto chunk_at = [&](int c) { return begin + (REV ? n - 1 - c : c) * kChunk; };
  request(chunk_at(0));
  State<R / 32> S;
  const float* first = f.seg_first ? f.seg_first + ((int64_t)head * a.nseg + seg) * D
                                   : (f.first ? f.first + head * D : nullptr);
  if (first) load_state(S.s, first, f.s_rs, f.s_cs, c0, lane);
  else S.clear();
  for (int c = 0; c < n; ++c) {
    const int t0 = chunk_at(c);
    __syncthreads();   // the last chunk's tiles are read, its dots written
    if constexpr (PAIR) {
      if (c > 0) sum_dots(chunk_at(c - 1));
    }
    gq.store(now.q, tid);
    gk.store(now.k, tid);
    gv.store(now.v, tid);
    if constexpr (PAIR) gy.store(now.y, tid);
    gd.store(now.dec, a.scale, tid);
    __syncthreads();
    if (c + 1 < n) request(chunk_at(c + 1));
    f32x16 o;
    const float dot = chunk_step<Tin, R, C, REV, PAIR>(now.q, now.k, now.v, now.y, now.dec, a.scale, c0, lane, S, o);
    if constexpr (PAIR) {
      if (lane < 32) now.dots[wave][lane] = dot;
    }
    if (PAIR && f.out_f32)
      store_out(row_base<float>(f.out, b, h) + t0 * f.out.st, f.out.st, c0, o, lim - t0, end - t0, lane);
    else
      store_out(row_base<Tin>(f.out, b, h) + t0 * f.out.st, f.out.st, c0, o, lim - t0, end - t0, lane);
  }
  if constexpr (PAIR) {
    __syncthreads();
    sum_dots(chunk_at(n - 1));
  }
  if (seg == (REV ? 0 : a.nseg - 1)) {
    S.apply();
    if (f.last) store_state(S.s, f.last + head * D, f.s_rs, f.s_cs, c0, lane);
    if constexpr (PAIR) {
      if (f.end_with) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < R / 32; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            x += S.s[i][r] * f.end_with[head * D + (32 * i + held_row(r, lane)) * f.s_rs +
                                        (c0 + perm_row(lane & 31)) * f.s_cs];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
        __syncthreads();
        if (lane == 0) now.dots[wave][0] = x;
        __syncthreads();
        if (tid == 0) {
          float z = 0.f;
          for (int w = 0; w < NW; ++w) z += now.dots[w][0];
          f.end_dot[head] = z;
        }
      }
    }
  }
}

// A segment's own part of the state behind it, sum over its tokens of (decay to the
// segment's end) k_s v_s^T; reverse: of the adjoint before it, sum of scale (decay from
// the segment's start) q_s do_s^T.  Both go from the segment's last chunk to its first: the
// pass that follows begins there, with what is still in the caches.  Going back the state
// itself does not decay, each chunk's part does, and where nothing is left of it (a cut
// gate behind it) the rest of the segment adds nothing and is not read.
template <typename Tin, int DK, int DV>
struct SegTiles {
  Tin k[Tile<Tin, DK>::SIZE], v[Tile<Tin, DV>::SIZE];
  float in[kChunk], out[kChunk];
};

template <typename Tin, int DK, int DV, bool REV>
__global__ __launch_bounds__(2 * DV, sizeof(Tin) == 4 ? 1 : (DV == 128 ? 3 : 2)) void segment_kernel(RecArgs a, Rows xr, Rows yr, float* dst) {
  constexpr int NT = 2 * DV, ST = DK / 32;
  __shared__ __align__(16) SegTiles<Tin, DK, DV> tiles[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H, c0 = 32 * wave;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const Tin* x = row_base<const Tin>(xr, b, h);
  const Tin* y = row_base<const Tin>(yr, b, h);
  const int64_t padded = rec_padded(a.T);
  const float2* decays = a.decays + 2 * head * padded + padded;
  State<ST> S;
  S.clear();
  float decay = 1.f;
  Stage<Tin, DK, NT> gx;
  Stage<Tin, DV, NT> gy;
  float2 gd;
  auto request = [&](int t0) {
    gx.load(x + t0 * xr.st, xr.st, lim - t0, tid);
    gy.load(y + t0 * yr.st, yr.st, lim - t0, tid);
    if (tid < kChunk) gd = decays[t0 + tid];
  };
  auto store = [&](SegTiles<Tin, DK, DV>& to) {
    gx.store(to.k, tid);
    gy.store(to.v, tid);
    if (tid < kChunk) {
      to.in[tid] = gd.x;
      to.out[tid] = gd.y;
    }
  };
  const int n = (end - begin + kChunk - 1) / kChunk;
  auto chunk_at = [&](int c) { return begin + (n - 1 - c) * kChunk; };
  request(chunk_at(0));
  store(tiles[0]);
  __syncthreads();
  for (int c = 0; c < n; ++c) {
    const SegTiles<Tin, DK, DV>& now = tiles[c & 1];
    if (c + 1 < n) request(chunk_at(c + 1));
    const float total = now.in[kChunk - 1];
    if (REV && S.decay(total)) S.apply();
    const float weight = REV ? a.scale * __builtin_amdgcn_rcpf(S.f) : decay;
    decay = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(decay * total)));
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      float w[8];
      weights8(REV ? now.in : now.out, kk, lane, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] *= weight;
      const Scaled<Tin> z(Tile<Tin, DV>::col_frag(now.v, c0, kk, lane), w);
#pragma unroll
      for (int i = 0; i < ST; ++i) z.mma_b(S.s[i], Tile<Tin, DK>::col_frag(now.k, 32 * i, kk, lane));
    }
    if (!REV && decay == 0.f) break;
    if (c + 1 < n) store(tiles[(c + 1) & 1]);
    __syncthreads();
  }
  S.apply();
  store_state(S.s, dst + ((int64_t)head * a.nseg + seg) * DK * DV, DV, 1, c0, lane);
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

template <bool REV, bool PAIR>
hipError_t launch_scan(const ScanArgs& f, int dtype, int R, int C, hipStream_t st) {
  const dim3 grid(f.a.B * f.a.H * f.a.nseg), block(2 * C);
  if (dtype == DLA_BF16) {
    if (R == 128 && C == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 128, 128, REV, PAIR>), grid, block, 0, st, f);
    else if (R == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 128, 64, REV, PAIR>), grid, block, 0, st, f);
    else if (C == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 64, 128, REV, PAIR>), grid, block, 0, st, f);
    else hipLaunchKernelGGL((scan_kernel<bf16_t, 64, 64, REV, PAIR>), grid, block, 0, st, f);
  } else {
    if (R == 128 && C == 128) hipLaunchKernelGGL((scan_kernel<float, 128, 128, REV, PAIR>), grid, block, 0, st, f);
    else if (R == 128) hipLaunchKernelGGL((scan_kernel<float, 128, 64, REV, PAIR>), grid, block, 0, st, f);
    else if (C == 128) hipLaunchKernelGGL((scan_kernel<float, 64, 128, REV, PAIR>), grid, block, 0, st, f);
    else hipLaunchKernelGGL((scan_kernel<float, 64, 64, REV, PAIR>), grid, block, 0, st, f);
  }
  return hipGetLastError();
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
  ScanArgs f{};
  f.a = a;
  f.q = q;
  f.k = k;
  f.v = v;
  f.out = out;
  f.first = s0;
  f.s_rs = a.dv;
  f.s_cs = 1;
  f.seg_first = a.nseg > 1 ? a.seg_state : nullptr;
  f.last = s_out;
  return launch_scan<false, false>(f, dtype, a.dk, a.dv, st);
}

hipError_t launch_recurrence_dq(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                const Rows& v, const Rows& dout, const Rows& dq, bool dq_f32,
                                const float* s0, const float* dstate, float* qdot, float* end_dot,
                                hipStream_t st) {
  ScanArgs f{};
  f.a = a;
  f.q = dout;
  f.k = v;
  f.v = k;
  f.out = dq;
  f.y = q;
  f.first = s0;
  f.s_rs = 1;
  f.s_cs = a.dv;
  f.seg_first = a.nseg > 1 ? a.seg_state : nullptr;
  f.dot = qdot;
  f.end_with = dstate;
  f.end_dot = end_dot;
  f.out_f32 = dq_f32 ? 1 : 0;
  return launch_scan<false, true>(f, dtype, a.dv, a.dk, st);
}

hipError_t launch_recurrence_adjoint(const RecArgs& a, int dtype, const Rows& q, const Rows& k,
                                     const Rows& v, const Rows& dout, const Rows& dk, bool dk_f32,
                                     const Rows& dv, const float* dstate, float* ds0, float* kdot,
                                     hipStream_t st) {
  // dk before dv, so that ds0, which the latter writes, may be dstate's array
  ScanArgs f{};
  f.a = a;
  f.q = v;
  f.k = dout;
  f.v = q;
  f.out = dk;
  f.y = k;
  f.first = dstate;
  f.s_rs = 1;
  f.s_cs = a.dv;
  f.seg_first = a.nseg > 1 ? a.seg_adj : nullptr;
  f.dot = kdot;
  f.out_f32 = dk_f32 ? 1 : 0;
  const hipError_t e = launch_scan<true, true>(f, dtype, a.dv, a.dk, st);
  if (e != hipSuccess) return e;
  f.q = k;
  f.k = q;
  f.v = dout;
  f.out = dv;
  f.y = Rows();
  f.s_rs = a.dv;
  f.s_cs = 1;
  f.last = ds0;
  f.dot = nullptr;
  f.out_f32 = 0;
  return launch_scan<true, false>(f, dtype, a.dk, a.dv, st);
}

}  // namespace dla
