// The single-state recurrence over long sequences, and dq, dk and dv of its backward pass.
//
// A workgroup takes one head's segment of tokens, a chunk at a time (recurrence_tile.h
// has the chunk's formulas).  Wave w holds columns 32 w .. 32 w + 31 of the state, all
// d_k rows of them, in the accumulators of the products that update it; their layout is
// that of the first operand of the product that reads them, so the state never leaves
// the registers.  The chunk's scores are formed once, 16 x 16 of them a wave, and go through
// LDS to all waves, which meet only after the state's products (4 x 16k tokens of 16 heads,
// forward and backward: 1514 us when each wave formed them all for itself, 1415 so).
//
// The backward pass is the same kernel with other roles (a_t, a_end as in recurrence_tile.h):
//   dq_t = e^{a_t} S do_t + scale sum_{s <= t} e^{a_t - a_s} (do_t . v_s) k_s
// with do, v and k in the places of q, k and v and the state transposed; and, back in time,
// with R the adjoint of the state behind a chunk (what later tokens and the last state's
// gradient ask of it),
//   dv_s = e^{a_end - a_s} R^T k_s + scale sum_{u >= s} e^{a_u - a_s} (q_u . k_s) do_u
//   dk_s = e^{a_end - a_s} R v_s   + scale sum_{u >= s} e^{a_u - a_s} (do_u . v_s) q_u
//   R   <- e^{a_end} R + scale sum_u e^{a_u} q_u do_u^T.
// The passes of dq and dk also leave what pairs of tokens give to the gates between them
// (recurrence_grad.hip).
//
// What bounds it.  Forward, 4 x 16 heads x 16k tokens of 128 x 128 bfloat16: 234 us for 1.07
// GB, 4.6 TB/s (a large copy 5.1), after 123 for the segments' states (0.54 GB).  dq: 326 us
// for 1.34 GB, 4.1 TB/s; dk and dv: 528 us for 1.6 GB, the chunk's own chain of LDS reads,
// products and arithmetic at two waves a SIMD.  A third wave in the forward pass takes 17
// registers through scratch memory (300 heads x 2k tokens 172 -> 239 us).  Of repeated calls
// the first is faster (dk and dv 473 us): the clock falls under load, so what counts is the
// number of instructions rather than their latency.
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
  Scores<Tin> p;
  float dots[2][PAIR ? C / 32 + 2 : 1][kChunk];   // of the chunk at hand and the one before
};

// REV: from the segment's last chunk to its first.  (REV is float32's; bfloat16's dk and dv
// come from adjoint_kernel.)
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
  const int n = (end - begin + kChunk - 1) / kChunk;
  const int t_first = REV ? begin + (n - 1) * kChunk : begin;
  constexpr int STEP = REV ? -kChunk : kChunk;
  const int64_t D = (int64_t)R * C, padded = rec_padded(a.T);
  // the addresses of the next chunk to load, and of the next one's outputs
  const Tin* q = row_base<const Tin>(f.q, b, h) + t_first * f.q.st;
  const Tin* k = row_base<const Tin>(f.k, b, h) + t_first * f.k.st;
  const Tin* v = row_base<const Tin>(f.v, b, h) + t_first * f.v.st;
  const Tin* y = PAIR ? row_base<const Tin>(f.y, b, h) + t_first * f.y.st : nullptr;
  const float2* decays = a.decays + 2 * head * padded + t_first;
  char* out = static_cast<char*>(f.out.p) +
              (b * f.out.sb + (h / f.out.hdiv) * f.out.sh + t_first * f.out.st) * (PAIR && f.out_f32 ? 4 : sizeof(Tin));
  float* dot_out = PAIR ? f.dot + (int64_t)head * a.T : nullptr;

  Stage<Tin, R, NT> gq, gk;
  Stage<Tin, C, NT> gv, gy;
  DecayStage gd;
  auto request = [&](int t0) {
    gq.load(q, f.q.st, lim - t0, tid);
    gk.load(k, f.k.st, lim - t0, tid);
    gv.load(v, f.v.st, lim - t0, tid);
    if constexpr (PAIR) gy.load(y, f.y.st, lim - t0, tid);
    gd.load(decays, padded, tid);
    q += STEP * f.q.st;
    k += STEP * f.k.st;
    v += STEP * f.v.st;
    if constexpr (PAIR) y += STEP * f.y.st;
    decays += STEP;
  };
  // a chunk's dots, the sum of the waves' parts
  auto sum_dots = [&](int which, int t0) {
    if (tid < kChunk && t0 + tid < end) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < NW + 2; ++w) x += now.dots[which][w][tid];
      dot_out[t0 + tid] = t0 + tid < lim ? x : 0.f;
    }
  };
  request(t_first);
  State<R / 32> S;
  const float* first = f.seg_first ? f.seg_first + ((int64_t)head * a.nseg + seg) * D
                                   : (f.first ? f.first + head * D : nullptr);
  if (first) load_state(S.s, first, f.s_rs, f.s_cs, c0, lane);
  else S.clear();
  int t0 = t_first;
  for (int c = 0; c < n; ++c, t0 += STEP) {
    __syncthreads();   // the last chunk's tiles are read, its dots written
    gq.store(now.q, tid);
    gk.store(now.k, tid);
    gv.store(now.v, tid);
    if constexpr (PAIR) gy.store(now.y, tid);
    gd.store(now.dec, tid);
    __syncthreads();
    if (c + 1 < n) request(t0 + STEP);
    if constexpr (PAIR) {
      if (c > 0) sum_dots((c - 1) & 1, t0 - STEP);
    }
    // scores, a quarter (NW = 2: a half) a wave
#pragma unroll
    for (int i = wave; i < 4; i += NW) {
      const int th = 16 * (i & 1), sh = 16 * (i >> 1);
      f32x4 p = {0.f, 0.f, 0.f, 0.f};
      float x = 0.f;
      if (REV ? sh >= th : sh <= th) {
        p = scores16<Tin, R>(now.k, now.q, sh, th, lane) * decays16<REV>(now.dec, a.scale, sh, th, lane);
        if constexpr (PAIR) x = pairs16(p, scores16<Tin, C>(now.v, now.y, sh, th, lane), sh, th, lane);
      }
      now.p.put(th + (lane & 15), sh + 4 * (lane >> 4), p);
      if constexpr (PAIR) {
        if (lane < 16) now.dots[c & 1][NW + (i >> 1)][th + lane] = x;
      }
    }
    f32x16 o;
    const float dot = chunk_step<Tin, R, C, REV, PAIR>(now.q, now.k, now.v, now.y, now.dec, now.p, a.scale, c0, lane, S, o);
    if constexpr (PAIR) {
      if (lane < 32) now.dots[c & 1][wave][lane] = dot;
    }
    if (PAIR && f.out_f32) {
      store_out(reinterpret_cast<float*>(out), f.out.st, c0, o, lim - t0, end - t0, lane);
      out += STEP * f.out.st * 4;
    } else {
      store_out(reinterpret_cast<Tin*>(out), f.out.st, c0, o, lim - t0, end - t0, lane);
      out += STEP * f.out.st * (int)sizeof(Tin);
    }
  }
  if constexpr (PAIR) {
    __syncthreads();
    sum_dots((n - 1) & 1, t0 - STEP);
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
        if (lane == 0) now.dots[0][wave][0] = x;
        __syncthreads();
        if (tid == 0) {
          float z = 0.f;
          for (int w = 0; w < NW; ++w) z += now.dots[0][w][0];
          f.end_dot[head] = z;
        }
      }
    }
  }
}

// dk and dv at once: half of the waves hold the adjoint's columns and give dv, the others
// those of its transpose and give dk, from the same tiles.  A chunk's tokens are read once
// for both, and its next one is stored into the other set of tiles meanwhile.  Against two
// passes of scan_kernel, 2k tokens forward and backward: 200 heads 496 us against 587, 512
// heads (two rounds of workgroups) 993 against 1080, 16 heads 129 against 138.
// float32 does not fit: its operands are twice as wide, and the waves' registers spill.
template <typename Tin, int DK, int DV>
struct AdjointTiles {
  Tin q[Tile<Tin, DK>::SIZE], k[Tile<Tin, DK>::SIZE], v[Tile<Tin, DV>::SIZE], o[Tile<Tin, DV>::SIZE];
  Decays dec;
  float dots[DK / 32 + 2][kChunk];
};

struct AdjointArgs {
  RecArgs a;
  Rows q, k, v, dout, dk, dv;
  const float* dstate;
  float* ds0;
  float* kdot;
  int dk_f32;
};

template <typename Tin, int DK, int DV>
__global__ __launch_bounds__(2 * (DK + DV), 2) void adjoint_kernel(AdjointArgs f) {
  constexpr int NT = 2 * (DK + DV), KW = DK / 32, VW = DV / 32;
  __shared__ __align__(16) AdjointTiles<Tin, DK, DV> tiles[2];
  __shared__ __align__(16) Scores<Tin> scores[2];   // of q and k, for dv; of dout and v, for dk
  const RecArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % (a.B * a.H), seg = blockIdx.x / (a.B * a.H);
  const int b = head / a.H, h = head % a.H;
  const int lim = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int begin = seg * a.seg_len, end = min(a.T, begin + a.seg_len);
  const int t_last = begin + (end - begin - 1) / kChunk * kChunk;
  const int64_t D = (int64_t)DK * DV, padded = rec_padded(a.T);
  const Tin* q = row_base<const Tin>(f.q, b, h) + t_last * f.q.st;
  const Tin* k = row_base<const Tin>(f.k, b, h) + t_last * f.k.st;
  const Tin* v = row_base<const Tin>(f.v, b, h) + t_last * f.v.st;
  const Tin* o = row_base<const Tin>(f.dout, b, h) + t_last * f.dout.st;
  const float2* decays = a.decays + 2 * head * padded + t_last;
  Stage<Tin, DK, NT> gq, gk;
  Stage<Tin, DV, NT> gv, go;
  DecayStage gd;
  auto request = [&](int t0) {
    gq.load(q, f.q.st, lim - t0, tid);
    gk.load(k, f.k.st, lim - t0, tid);
    gv.load(v, f.v.st, lim - t0, tid);
    go.load(o, f.dout.st, lim - t0, tid);
    gd.load(decays, padded, tid);
    q -= kChunk * f.q.st;
    k -= kChunk * f.k.st;
    v -= kChunk * f.v.st;
    o -= kChunk * f.dout.st;
    decays -= kChunk;
  };
  auto store = [&](AdjointTiles<Tin, DK, DV>& to) {
    gq.store(to.q, tid);
    gk.store(to.k, tid);
    gv.store(to.v, tid);
    go.store(to.o, tid);
    gd.store(to.dec, tid);
  };
  const float* last = a.nseg > 1 ? a.seg_adj + ((int64_t)head * a.nseg + seg) * D
                                 : (f.dstate ? f.dstate + head * D : nullptr);
  request(t_last);
  int at = 0;
  if (wave < VW) {
    const int c0 = 32 * wave;
    State<DK / 32> R;
    if (last) load_state(R.s, last, DV, 1, c0, lane);
    else R.clear();
    store(tiles[0]);
    __syncthreads();
    Tin* out = row_base<Tin>(f.dv, b, h) + t_last * f.dv.st;
    for (int t0 = t_last; t0 >= begin; t0 -= kChunk, at ^= 1) {
      AdjointTiles<Tin, DK, DV>& now = tiles[at];
      if (t0 > begin) request(t0 - kChunk);
      // dv's waves have less to do: both kinds of scores, and the pairs' sums
#pragma unroll
      for (int i = wave; i < 4; i += VW) {
        const int th = 16 * (i & 1), sh = 16 * (i >> 1);
        f32x4 p = {0.f, 0.f, 0.f, 0.f}, z = p;
        float sum = 0.f;
        if (sh >= th) {
          const f32x4 d = decays16<true>(now.dec, a.scale, sh, th, lane);
          p = scores16<Tin, DK>(now.q, now.k, sh, th, lane);
          z = scores16<Tin, DV>(now.o, now.v, sh, th, lane) * d;
          sum = pairs16(z, p, sh, th, lane);
          p *= d;
        }
        scores[0].put(th + (lane & 15), sh + 4 * (lane >> 4), p);
        scores[1].put(th + (lane & 15), sh + 4 * (lane >> 4), z);
        if (lane < 16) now.dots[KW + (i >> 1)][th + lane] = sum;
      }
      f32x16 x;
      chunk_step<Tin, DK, DV, true, false>(now.k, now.q, now.o, nullptr, now.dec, scores[0], a.scale, c0, lane, R, x);
      store_out(out, f.dv.st, c0, x, lim - t0, end - t0, lane);
      out -= kChunk * f.dv.st;
      if (t0 > begin) store(tiles[at ^ 1]);
      __syncthreads();
    }
    // dk's waves have read dstate before the first barrier: ds0 may be its array
    if (seg == 0 && f.ds0) {
      R.apply();
      store_state(R.s, f.ds0 + head * D, DV, 1, c0, lane);
    }
  } else {
    const int c0 = 32 * (wave - VW);
    State<DV / 32> R;
    if (last) load_state(R.s, last, 1, DV, c0, lane);
    else R.clear();
    float* dot_out = f.kdot + (int64_t)head * a.T;
    auto sum_dots = [&](const AdjointTiles<Tin, DK, DV>& from, int t0) {
      if (c0 == 0 && lane < kChunk && t0 + lane < end) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < KW + 2; ++i) x += from.dots[i][lane];
        dot_out[t0 + lane] = t0 + lane < lim ? x : 0.f;
      }
    };
    store(tiles[0]);
    __syncthreads();
    char* out = static_cast<char*>(f.dk.p) +
                (b * f.dk.sb + (h / f.dk.hdiv) * f.dk.sh + t_last * f.dk.st) * (f.dk_f32 ? 4 : sizeof(Tin));
    for (int t0 = t_last; t0 >= begin; t0 -= kChunk, at ^= 1) {
      AdjointTiles<Tin, DK, DV>& now = tiles[at];
      if (t0 > begin) request(t0 - kChunk);
      if (t0 < t_last) sum_dots(tiles[at ^ 1], t0 + kChunk);
      f32x16 x;
      const float dot = chunk_step<Tin, DV, DK, true, true>(now.v, now.o, now.q, now.k, now.dec, scores[1], a.scale, c0, lane, R, x);
      if (lane < 32) now.dots[c0 / 32][lane] = dot;
      if (f.dk_f32) {
        store_out(reinterpret_cast<float*>(out), f.dk.st, c0, x, lim - t0, end - t0, lane);
        out -= kChunk * f.dk.st * 4;
      } else {
        store_out(reinterpret_cast<Tin*>(out), f.dk.st, c0, x, lim - t0, end - t0, lane);
        out -= kChunk * f.dk.st * (int)sizeof(Tin);
      }
      if (t0 > begin) store(tiles[at ^ 1]);
      __syncthreads();
    }
    sum_dots(tiles[at ^ 1], begin);
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
// them), four elements of a head's state per thread.  Reverse, also the products of the
// adjoint behind each segment but the last with the state there, which anchor the gates' sums
// (recurrence_grad.hip): a wave leaves the sum of its 256 elements.  Parts are read eight
// segments at a time, before any is replaced: 8 segments of 64 heads of 128 x 128 11 us and 17
// in reverse (one read after the other 14.5, and as much again 17 for the products apart).
template <bool REV>
__global__ __launch_bounds__(256) void prefix_kernel(RecArgs a, float* part, const float* first, double* anchor) {
  constexpr int NB = 8;
  const int64_t D4 = (int64_t)a.dk * a.dv / 4;
  const int head = blockIdx.y, lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;   // D4 is a multiple of 256
  float4* p = reinterpret_cast<float4*>(part) + (int64_t)head * a.nseg * D4 + i;
  const float4* state = reinterpret_cast<const float4*>(a.seg_state) + (int64_t)head * a.nseg * D4 + i;
  const float* decay = a.seg_decay + (int64_t)head * a.nseg;
  float4 cur = first ? reinterpret_cast<const float4*>(first)[head * D4 + i] : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j0 = 0; j0 < a.nseg; j0 += NB) {
    float4 own[NB], with[NB];
    float d[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {   // past the last segment: its part again, not used
      const int j = min(j0 + n, a.nseg - 1), s = REV ? a.nseg - 1 - j : j;
      own[n] = p[s * D4];
      d[n] = decay[s];
      if constexpr (REV) with[n] = state[min(s + 1, a.nseg - 1) * D4];
    }
    double x[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int j = j0 + n, s = REV ? a.nseg - 1 - j : j;
      if (j < a.nseg) p[s * D4] = cur;
      if constexpr (REV)
        x[n] = ((double)cur.x * with[n].x + (double)cur.y * with[n].y) +
               ((double)cur.z * with[n].z + (double)cur.w * with[n].w);
      cur.x = d[n] * cur.x + own[n].x;
      cur.y = d[n] * cur.y + own[n].y;
      cur.z = d[n] * cur.z + own[n].z;
      cur.w = d[n] * cur.w + own[n].w;
    }
    if constexpr (REV) {
      // eight sums over the wave at once: each step halves the lanes of a sum and the sums
      // of a lane, until lane 8 n holds sum n
#pragma unroll
      for (int o = 32, n = NB / 2; o >= 8; o >>= 1, n >>= 1) {
#pragma unroll
        for (int m = 0; m < n; ++m) {
          const bool up = lane & o;
          const double keep = up ? x[m + n] : x[m], give = up ? x[m] : x[m + n];
          x[m] = keep + __shfl_xor(give, o);
        }
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) x[0] += __shfl_xor(x[0], o);
      const int j = j0 + (lane >> 3);
      if ((lane & 7) == 0 && j > 0 && j < a.nseg)
        anchor[((int64_t)head * a.nseg + a.nseg - 1 - j) * (D4 / 64) + i / 64] = x[0];
    }
  }
}

template <bool REV, bool PAIR>
hipError_t launch_scan(const ScanArgs& f, int dtype, int R, int C, hipStream_t st) {
  const dim3 grid(f.a.B * f.a.H * f.a.nseg), block(2 * C);
  if (dtype == DLA_BF16) {
    if constexpr (!REV) {
      if (R == 128 && C == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 128, 128, false, PAIR>), grid, block, 0, st, f);
      else if (R == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 128, 64, false, PAIR>), grid, block, 0, st, f);
      else if (C == 128) hipLaunchKernelGGL((scan_kernel<bf16_t, 64, 128, false, PAIR>), grid, block, 0, st, f);
      else hipLaunchKernelGGL((scan_kernel<bf16_t, 64, 64, false, PAIR>), grid, block, 0, st, f);
    }
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
                        double* anchor, hipStream_t st) {
  const dim3 grid(a.B * a.H * a.nseg), block(2 * DV), pg(DK * DV / 1024, a.B * a.H);
  float* dst = rev ? a.seg_adj : a.seg_state;
  if (rev) {
    hipLaunchKernelGGL((segment_kernel<Tin, DK, DV, true>), grid, block, 0, st, a, x, y, dst);
    hipLaunchKernelGGL((prefix_kernel<true>), pg, dim3(256), 0, st, a, dst, first, anchor);
  } else {
    hipLaunchKernelGGL((segment_kernel<Tin, DK, DV, false>), grid, block, 0, st, a, x, y, dst);
    hipLaunchKernelGGL((prefix_kernel<false>), pg, dim3(256), 0, st, a, dst, first, anchor);
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
                                      const Rows& y, const float* first, double* anchor, hipStream_t st) {
  if (dtype == DLA_BF16) {
    if (a.dk == 128) return a.dv == 128 ? run_segments<bf16_t, 128, 128>(a, reverse, x, y, first, anchor, st) : run_segments<bf16_t, 128, 64>(a, reverse, x, y, first, anchor, st);
    return a.dv == 128 ? run_segments<bf16_t, 64, 128>(a, reverse, x, y, first, anchor, st) : run_segments<bf16_t, 64, 64>(a, reverse, x, y, first, anchor, st);
  }
  if (a.dk == 128) return a.dv == 128 ? run_segments<float, 128, 128>(a, reverse, x, y, first, anchor, st) : run_segments<float, 128, 64>(a, reverse, x, y, first, anchor, st);
  return a.dv == 128 ? run_segments<float, 64, 128>(a, reverse, x, y, first, anchor, st) : run_segments<float, 64, 64>(a, reverse, x, y, first, anchor, st);
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
  if (dtype == DLA_BF16) {
    const AdjointArgs f{a, q, k, v, dout, dk, dv, dstate, ds0, kdot, dk_f32 ? 1 : 0};
    const dim3 grid(a.B * a.H * a.nseg), block(2 * (a.dk + a.dv));
    if (a.dk == 128 && a.dv == 128) hipLaunchKernelGGL((adjoint_kernel<bf16_t, 128, 128>), grid, block, 0, st, f);
    else if (a.dk == 128) hipLaunchKernelGGL((adjoint_kernel<bf16_t, 128, 64>), grid, block, 0, st, f);
    else if (a.dv == 128) hipLaunchKernelGGL((adjoint_kernel<bf16_t, 64, 128>), grid, block, 0, st, f);
    else hipLaunchKernelGGL((adjoint_kernel<bf16_t, 64, 64>), grid, block, 0, st, f);
    return hipGetLastError();
  }
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
