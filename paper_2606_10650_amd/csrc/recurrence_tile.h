// What the recurrence's chunk kernels share: a chunk's tokens in LDS, its decays, and the
// products of a wave's columns of the state with them.
//
// With a_t the sum of the chunk's log decays up to and with token t, a chunk of tokens
// turns the state S before it into outputs and the state behind it by
//   o_t = e^{a_t} S^T q_t + sum_{s <= t} e^{a_t - a_s} (q_t . k_s) v_s
//   S  <- e^{a_end} S + sum_s e^{a_end - a_s} k_s v_s^T
// so everything but the state's own decay is a matrix product.  Every factor is the decay
// between two points in time, taken from a difference: nothing is divided by a decay, and
// none overflows where the gates are not above zero.
//
// A chunk is 32 tokens, one tile of scores: half of 64 x 64 scores' products lie beyond
// the mask or below it in tiles of their own, the state's products cost the same per token,
// and a wave's operands fit its registers twice over (64 tokens took 256 registers and
// spilled a hundred more).
#pragma once
#include "mfma.h"
#include "recurrence.h"

namespace dla {

constexpr int kChunk = 32;

// 32 rows of D values in LDS, in 16-byte pieces whose place in a row depends on the row,
// so that reads of one column by 16 rows, and of 64 (32: float32) bytes by the rows that
// one transposing read takes, spread over the banks.
template <typename Tin, int D>
struct Tile {
  static constexpr int PE = 16 / (int)sizeof(Tin);   // elements per piece
  static constexpr int NP = D / PE;                  // pieces per row
  __device__ static __forceinline__ int swz(int row) {
    if constexpr (sizeof(Tin) == 4) return row & 15;
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row << 1) & 4) | ((row >> 2) & 3);
  }
  __device__ static __forceinline__ int at(int row, int col) {
    return row * D + (((col / PE) ^ swz(row)) * PE) + col % PE;
  }
  // operand with a token per lane: row `row`, columns 16 kk + 8 (lane / 32) + e
  __device__ static __forceinline__ typename Frag<Tin>::T row_frag(const Tin* p, int row, int kk,
                                                                   int lane) {
    const int c = 16 * kk + 8 * (lane >> 5);
    if constexpr (sizeof(Tin) == 2) return Frag<Tin>::load(p + at(row, c));
    else return load_4x2<float>(p + at(row, c), p + at(row, c + 4));
  }
  // operand with a column per lane, c0 + perm_row(lane % 32), and tokens 16 kk + 8 (lane /
  // 32) + e
  __device__ static __forceinline__ typename Frag<Tin>::T col_frag(const Tin* p, int c0, int kk,
                                                                   int lane);
};

// Row of a product's first operand that lane m supplies: its output's elements 8 kk .. 8 kk
// + 7 are then the 8 consecutive rows 16 kk + 8 (lane / 32) + e, and the output serves as
// the next product's operand of a K = 16 step as it is.
__device__ __forceinline__ int perm_row(int m) {
  return (m & 16) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
}
__device__ __forceinline__ int held_row(int r, int lane) { return 16 * (r >> 3) + 8 * (lane >> 5) + (r & 7); }

template <typename Tin, int D>
__device__ __forceinline__ typename Frag<Tin>::T Tile<Tin, D>::col_frag(const Tin* p, int c0, int kk, int lane) {
  const int g = lane >> 5;
  if constexpr (sizeof(Tin) == 2) {
    // a 16-lane group reads 4 rows of 16 columns, 8 bytes a lane, and lane i gets column i
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const int i = lane & 15, c4 = i & 3;
    const int col = c0 + (lane & 16) + 8 * (c4 & 1) + 4 * (c4 >> 1);
    const int row = 16 * kk + 8 * g + (i >> 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + at(row, col)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + at(row + 4, col)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const int col = c0 + perm_row(lane & 31);
    f32x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = p[at(16 * kk + 8 * g + e, col)];
    return r;
  }
}

// A chunk's tokens on their way from memory into a tile: loads are issued into registers
// and stored later.  Rows from `lim` on are zero, whatever memory holds there.
template <typename Tin, int D, int NT>
struct Stage {
  using TL = Tile<Tin, D>;
  static constexpr int ALL = kChunk * TL::NP, N = (ALL + NT - 1) / NT;
  u32x4 v[N];
  __device__ __forceinline__ void load(const Tin* base, int64_t st, int t0, int lim, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = i * NT + tid, row = x / TL::NP, pc = x % TL::NP, t = t0 + row;
      v[i] = u32x4{0u, 0u, 0u, 0u};
      if ((ALL % NT == 0 || x < ALL) && t < lim)
        v[i] = *reinterpret_cast<const u32x4*>(base + t * st + pc * TL::PE);
    }
  }
  __device__ __forceinline__ void store(Tin* p, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = i * NT + tid, row = x / TL::NP, pc = x % TL::NP;
      if (ALL % NT == 0 || x < ALL) *reinterpret_cast<u32x4*>(p + TL::at(row, pc * TL::PE)) = v[i];
    }
  }
};

// A token's decays within its chunk.  In units of log2: a_t = hi + lo with hi whole, so
// that hi_t - hi_s is exact and the difference keeps float32's precision however large the
// sums are.  A gate whose decay is below float32's smallest normal number (-inf among them)
// cuts: it counts as a step of -2^17 in hi, which no sum of a chunk's other gates reaches.
// The decays kernel forms them once for all kernels of a call, float4 per token:
//   hi, lo, in = e^{a_t} (from before the chunk), out = e^{a_end - a_t} (to its end).
struct Decays {
  float hi[kChunk], lo[kChunk], in[kChunk], out[kChunk];
  __device__ __forceinline__ void store(const float4& d, int t) {
    hi[t] = d.x;
    lo[t] = d.y;
    in[t] = d.z;
    out[t] = d.w;
  }
  __device__ __forceinline__ float total() const { return in[kChunk - 1]; }   // e^{a_end}
};

__device__ __forceinline__ float decay2(float hi_t, float lo_t, float hi_s, float lo_s) {
  return __builtin_amdgcn_exp2f((hi_t - hi_s) + (lo_t - lo_s));
}

constexpr float kCutGate = -87.33655f;   // ln of 2^-126

// An operand scaled by float32 weights per k: for bfloat16 in two terms, whose sum keeps
// 16 bits or more of it, so that the states they add up to are not held to the 8 bits of one.
template <typename Tin>
struct Scaled;
template <>
struct Scaled<bf16_t> {
  bf16x8 h, l;
  __device__ __forceinline__ Scaled(const bf16x8& x, const float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = (float)x[e] * w[e];
      h[e] = (__bf16)y;
      l[e] = (__bf16)(y - (float)h[e]);
    }
  }
  __device__ __forceinline__ void mma_b(f32x16& acc, const bf16x8& a) const {
    Frag<bf16_t>::mma(acc, a, l);
    Frag<bf16_t>::mma(acc, a, h);
  }
};
template <>
struct Scaled<float> {
  f32x8 x;
  __device__ __forceinline__ Scaled(const f32x8& y, const float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e] * w[e];
  }
  __device__ __forceinline__ void mma_b(f32x16& acc, const f32x8& a) const { Frag<float>::mma(acc, a, x); }
};

// Eight of a chunk's per-token numbers, from token 16 kk + 8 (lane / 32)
__device__ __forceinline__ void weights8(const float* w, int kk, int lane, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(w + 16 * kk + 8 * (lane >> 5));
  const float4 b = *reinterpret_cast<const float4*>(w + 16 * kk + 8 * (lane >> 5) + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// A state tile as a product's first operand (lane: column, elements: rows), rounded once
// to the inputs' type; and what that rounding left.
template <typename Tin>
__device__ __forceinline__ typename Frag<Tin>::T state_frag(const f32x16& s, int kk) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = s[8 * kk + e];
  return Frag<Tin>::from_floats(x);
}
__device__ __forceinline__ bf16x8 state_frag_low(const f32x16& s, int kk, const bf16x8& h) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)(s[8 * kk + e] - (float)h[e]);
  return r;
}

// A wave's columns c0 .. c0 + 31 of a state of R rows (strides rs, cs): tile i holds rows
// 32 i + held_row(element), column c0 + perm_row(lane % 32).
template <int N>
__device__ __forceinline__ void load_state(f32x16 (&s)[N], const float* p, int64_t rs, int64_t cs, int c0, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      s[i][r] = p[(32 * i + held_row(r, lane)) * rs + (c0 + perm_row(lane & 31)) * cs];
}
template <int N>
__device__ __forceinline__ void store_state(const f32x16 (&s)[N], float* p, int64_t rs, int64_t cs, int c0, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      p[(32 * i + held_row(r, lane)) * rs + (c0 + perm_row(lane & 31)) * cs] = s[i][r];
}

// One chunk, for a wave's 32 columns of a state of R rows.  Lane l % 32 is token t; the
// elements of c and o are columns c0 + held_row(r).
//   p[r] = q_t . k_s with s = held_row(r)
//   c = carry_t S^T q_t
//   o = c + scale sum over s of p masked and decayed, times v_s
// and the state takes up the chunk.  REV: time runs back, so s >= t.  PAIR: c also
// takes what the state's rounding to bfloat16 leaves, and the lane's part of
//   dot_t = y_t . c + scale sum over s != t of p masked and decayed, times (y_t . v_s)
// is returned, with the rows y_t (32 columns of them a wave) in sy: what the pairs (s, t)
// give to the gates between them.
template <typename Tin, int R, int C, bool REV, bool PAIR>
__device__ __forceinline__ float chunk_step(const Tin* sq, const Tin* sk, const Tin* sv, const Tin* sy,
                                            const Decays& dec, float scale, int c0, int lane,
                                            f32x16 (&S)[R / 32], f32x16& o) {
  using F = typename Frag<Tin>::T;
  using TR = Tile<Tin, R>;
  using TC = Tile<Tin, C>;
  const int t = lane & 31, g = lane >> 5, kr = perm_row(t);
  const float hi = dec.hi[t], lo = dec.lo[t], total = dec.total();
  f32x16 p = zero16();
  o = zero16();
#pragma unroll
  for (int kk = 0; kk < R / 16; ++kk) {
    const F q = TR::row_frag(sq, t, kk, lane);
    Frag<Tin>::mma(p, TR::row_frag(sk, kr, kk, lane), q);
    const F s = state_frag<Tin>(S[kk >> 1], kk & 1);
    if constexpr (PAIR && sizeof(Tin) == 2) Frag<Tin>::mma(o, state_frag_low(S[kk >> 1], kk & 1, s), q);
    Frag<Tin>::mma(o, s, q);
  }
  // the scores, masked and decayed
  float w[2][8];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    float hs[8], ls[8];
    weights8(dec.hi, kk, lane, hs);
    weights8(dec.lo, kk, lane, ls);
    weights8(REV ? dec.in : dec.out, kk, lane, w[kk]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * kk + 8 * g + e;
      const float d = REV ? decay2(hs[e], ls[e], hi, lo) : decay2(hi, lo, hs[e], ls[e]);
      p[8 * kk + e] = (REV ? s >= t : s <= t) ? p[8 * kk + e] * d * scale : 0.f;
      if constexpr (REV) w[kk][e] *= scale;
    }
  }
  const float carry = REV ? dec.out[t] : dec.in[t] * scale;
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] *= carry;
  float dot = 0.f;
  if constexpr (PAIR) {
    f32x16 z = zero16();
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const F y = TC::row_frag(sy, t, c0 / 16 + kk, lane);
      Frag<Tin>::mma(z, TC::row_frag(sv, kr, c0 / 16 + kk, lane), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += o[8 * kk + e] * (float)y[e];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) dot += held_row(r, lane) != t ? p[r] * z[r] : 0.f;
    dot += __shfl_xor(dot, 32);
  }
#pragma unroll
  for (int i = 0; i < R / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[i][r] *= total;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[8 * kk + e];
    const F v = TC::col_frag(sv, c0, kk, lane);
    Frag<Tin>::mma(o, v, Frag<Tin>::from_floats(x));
    const Scaled<Tin> y(v, w[kk]);
#pragma unroll
    for (int i = 0; i < R / 32; ++i) y.mma_b(S[i], TR::col_frag(sk, 32 * i, kk, lane));
  }
  return dot;
}

// Eight consecutive values of an output row, rounded once to the output's type.
__device__ __forceinline__ void store8(bf16_t* p, const f32x16& x, int k) {
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[8 * k + e];
  *reinterpret_cast<bf16x8*>(p) = y;
}
__device__ __forceinline__ void store8(float* p, const f32x16& x, int k) {
  *reinterpret_cast<float4*>(p) = make_float4(x[8 * k], x[8 * k + 1], x[8 * k + 2], x[8 * k + 3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[8 * k + 4], x[8 * k + 5], x[8 * k + 6], x[8 * k + 7]);
}
// A lane's columns of its token's output row
template <typename Tout>
__device__ __forceinline__ void store_out(Tout* row, int c0, const f32x16& o, int lane) {
#pragma unroll
  for (int k = 0; k < 2; ++k) store8(row + c0 + 16 * k + 8 * (lane >> 5), o, k);
}

}  // namespace dla
