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
// A chunk is 32 tokens, one tile of scores: the state's products cost the same per token at
// any chunk length, and a wave's operands fit its registers (64 tokens took 256 of them and
// spilled a hundred more: 4 x 16k tokens forward and backward 5.5 ms, 1.7 with 32).
#pragma once
#include "mfma.h"
#include "recurrence.h"

namespace dla {

constexpr int kChunk = 32;

// 32 rows of D values in LDS, read a row per lane (16 bytes a lane) and a column per lane
// (bfloat16: 4 rows of 64 bytes per 16 lanes, transposed by the read; float32: 128 bytes of
// two rows, 8 apart).  bfloat16 rows are padded by 64 bytes, which spreads four rows over
// the banks, and pieces of 16 bytes change places within 64 bytes by bits 2 and 3 of the row,
// which spreads sixteen; float32 rows are padded by 16 bytes.  Both kinds of read are then
// free of conflicts (those of 16 x 16 scores, four pieces of sixteen rows, are not quite: with
// them conflicts take a seventh of the forward pass's LDS cycles), and but for those two bits
// every offset is a constant of the instruction.
template <typename Tin, int D>
struct Tile {
  static constexpr int PE = 16 / (int)sizeof(Tin);             // elements per piece
  static constexpr int NP = D / PE;                            // pieces per row
  static constexpr int LD = D + (sizeof(Tin) == 2 ? 32 : 4);   // elements from row to row
  static constexpr int SIZE = kChunk * LD;
  __device__ static __forceinline__ int swz(int row) { return sizeof(Tin) == 2 ? (row >> 2) & 3 : 0; }
  __device__ static __forceinline__ int at(int row, int col) {
    return row * LD + ((col / PE) ^ swz(row)) * PE + col % PE;
  }
  // operand with a token per lane: row `row`, columns 16 kk + 8 (lane / 32) + e
  __device__ static __forceinline__ typename Frag<Tin>::T row_frag(const Tin* p, int row, int kk,
                                                                   int lane) {
    return Frag<Tin>::load(p + at(row, 16 * (kk & 1) + 8 * (lane >> 5)) + 32 * (kk >> 1));
  }
  // operand of a 16 x 16 product: row `row` per lane % 16, columns 32 k + 8 (lane / 16) + e
  __device__ static __forceinline__ typename Frag<Tin>::T row_frag16(const Tin* p, int row, int k, int lane) {
    return Frag<Tin>::load(p + at(row, 8 * (lane >> 4)) + 32 * k);
  }
  // operand with a column per lane, c0 + perm_row(lane % 32) (c0 a multiple of 32), and
  // tokens 16 kk + 8 (lane / 32) + e
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
    const int row = 8 * g + (i >> 2), col = (lane & 16) + 8 * (c4 & 1) + 4 * (c4 >> 1);
    const Tin* x = p + 16 * kk * LD + c0;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(x + at(row, col)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(x + at(row + 4, col)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const Tin* x = p + at(8 * g, perm_row(lane & 31)) + 16 * kk * LD + c0;
    f32x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e * LD];
    return r;
  }
}

// A chunk's tokens on their way from memory into a tile: loads are issued into registers
// and stored later.  `chunk` is the address of the chunk's first row, the same for all
// threads; rows from n on are zero, whatever memory holds there.
template <typename Tin, int D, int NT>
struct Stage {
  using TL = Tile<Tin, D>;
  static constexpr int STEP = NT / TL::NP;                      // rows per pass
  static constexpr int N = (kChunk + STEP - 1) / STEP;
  static_assert(NT % TL::NP == 0, "whole rows per pass");
  u32x4 v[N];
  __device__ __forceinline__ void load(const Tin* chunk, int64_t st, int n, int tid) {
    const uint32_t row = tid / TL::NP, off = row * (uint32_t)st + (tid % TL::NP) * TL::PE;
    if (n >= kChunk && kChunk % STEP == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const u32x4*>(chunk + i * STEP * st + off);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = u32x4{0u, 0u, 0u, 0u};
        if (i * STEP + (int)row < min(n, kChunk))
          v[i] = *reinterpret_cast<const u32x4*>(chunk + i * STEP * st + off);
      }
    }
  }
  __device__ __forceinline__ void store(Tin* p, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = i * STEP + tid / TL::NP;
      if (kChunk % STEP == 0 || row < kChunk)
        *reinterpret_cast<u32x4*>(p + TL::at(row, tid % TL::NP * TL::PE)) = v[i];
    }
  }
};

// A token's decays within its chunk.  In units of log2: a_t = hi + lo with hi whole, so
// that hi_t - hi_s is exact and the difference keeps float32's precision however large the
// sums are.  A gate whose decay is below float32's smallest normal number (-inf among them)
// cuts: it counts as a step of -2^17 in hi, which no sum of a chunk's other gates reaches.
// The decays kernel forms them once for all kernels of a call, per head hi and lo of every
// token, then
//   in = e^{a_t} (from before the chunk) and out = e^{a_end - a_t} (to its end) of every token.
__device__ __forceinline__ float decay2(float hi_t, float lo_t, float hi_s, float lo_s) {
  return __builtin_amdgcn_exp2f((hi_t - hi_s) + (lo_t - lo_s));
}

// A chunk's decays in LDS: in and out, and a_t as hi and lo for those between its tokens.
struct Decays {
  float in[kChunk], out[kChunk];
  float2 at[kChunk];
  __device__ __forceinline__ float total() const { return in[kChunk - 1]; }   // e^{a_end}
};

// On its way from memory, by the first threads.
struct DecayStage {
  float2 io, t;
  // chunk: the first token's hi and lo; its in and out are `padded` behind
  __device__ __forceinline__ void load(const float2* chunk, int64_t padded, int tid) {
    if (tid < kChunk) {
      t = chunk[tid];
      io = chunk[padded + tid];
    }
  }
  __device__ __forceinline__ void store(Decays& d, int tid) const {
    if (tid < kChunk) {
      d.in[tid] = io.x;
      d.out[tid] = io.y;
      d.at[tid] = t;
    }
  }
};

// An operand scaled by float32 weights per k: for bfloat16 in two terms, whose sum keeps
// 16 bits or more of it, so that the states they add up to are not held to the 8 bits of one.
template <typename Tin>
struct Scaled;
template <>
struct Scaled<bf16_t> {
  bf16x8 h, l;
  __device__ __forceinline__ Scaled(const bf16x8& x, const float (&w)[8]) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = (float)x[e] * w[e];
      h[e] = (__bf16)y[e];
    }
    const u32x4 z = __builtin_bit_cast(u32x4, h);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      l[e] = (__bf16)(y[e] - __uint_as_float(z[e >> 1] << 16));
      l[e + 1] = (__bf16)(y[e + 1] - __uint_as_float(z[e >> 1] & 0xFFFF0000u));
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

// A state or score tile as a product's operand, rounded once to the inputs' type; and what
// that rounding left.
template <typename Tin>
__device__ __forceinline__ typename Frag<Tin>::T state_frag(const f32x16& s, int kk) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = s[8 * kk + e];
  return Frag<Tin>::from_floats(x);
}
__device__ __forceinline__ bf16x8 state_frag_low(const f32x16& s, int kk, const bf16x8& h) {
  const u32x4 w = __builtin_bit_cast(u32x4, h);   // by words: element by element each is rounded again
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    r[e] = (__bf16)(s[8 * kk + e] - __uint_as_float(w[e >> 1] << 16));
    r[e + 1] = (__bf16)(s[8 * kk + e + 1] - __uint_as_float(w[e >> 1] & 0xFFFF0000u));
  }
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

// A wave's columns of a state, as f times its tiles: a chunk's decay goes to the factor,
// and to the tiles only when that has become small, which saves a pass over them per chunk.
template <int N>
struct State {
  f32x16 s[N];
  float f = 1.f;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = zero16();
  }
  // Takes a decay, the same in all lanes (and known to be so: the factor is kept, and
  // branches on it are taken, once).  True if the factor has left 2^-16 .. 2^16, inside of
  // which what is added to the tiles, divided by it, stays well inside float32.
  __device__ __forceinline__ bool decay(float total) {
    f = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(f * total)));
    return !(f >= 1.52587890625e-05f && f <= 65536.f);
  }
  __device__ __forceinline__ void apply() {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[i][r] *= f;
    f = 1.f;
  }
};

// Masked and decayed scores of a chunk, [t][s], for the product with the values: bfloat16 in
// two terms (two more of some thirty products, and outputs of short sequences lose 2^-9
// instead of 2^-8.5).  Rows are padded by 16 bytes, which spreads them over the banks.
template <typename Tin>
struct Scores;
template <>
struct Scores<bf16_t> {
  static constexpr int LD = kChunk + 8, TERMS = 2;
  bf16_t x[2][kChunk * LD];
  __device__ __forceinline__ void put(int t, int s, const f32x4& p) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[e] = (__bf16)p[e];
      l[e] = (__bf16)(p[e] - (float)h[e]);
    }
    *reinterpret_cast<bf16x4*>(x[0] + t * LD + s) = h;
    *reinterpret_cast<bf16x4*>(x[1] + t * LD + s) = l;
  }
  __device__ __forceinline__ bf16x8 frag(int term, int t, int s) const {
    return Frag<bf16_t>::load(x[term] + t * LD + s);
  }
};
template <>
struct Scores<float> {
  static constexpr int LD = kChunk + 4, TERMS = 1;
  float x[kChunk * LD];
  __device__ __forceinline__ void put(int t, int s, const f32x4& p) {
    *reinterpret_cast<f32x4*>(x + t * LD + s) = p;
  }
  __device__ __forceinline__ f32x8 frag(int, int t, int s) const { return Frag<float>::load(x + t * LD + s); }
};

// 16 x 16 scores: lane l holds a . b of rows s0 + 4 (l / 16) + r of a and row t0 + l % 16 of b.
template <typename Tin, int D>
__device__ __forceinline__ f32x4 scores16(const Tin* a, const Tin* b, int s0, int t0, int lane) {
  using TL = Tile<Tin, D>;
  f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
    mma16(p, TL::row_frag16(a, s0 + (lane & 15), k, lane), TL::row_frag16(b, t0 + (lane & 15), k, lane));
  return p;
}
// scale times the decays between their tokens: from s to t, or with REV from t to s, zero
// where the later of a pair should come first.
template <bool REV>
__device__ __forceinline__ f32x4 decays16(const Decays& dec, float scale, int s0, int t0, int lane) {
  const int t = t0 + (lane & 15), s = s0 + 4 * (lane >> 4);
  const float2 x = dec.at[t];
  f32x4 d;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float2 y = dec.at[s + r];
    const float e = REV ? decay2(y.x, y.y, x.x, x.y) : decay2(x.x, x.y, y.x, y.y);
    d[r] = (REV ? s + r >= t : s + r <= t) ? e * scale : 0.f;
  }
  return d;
}
// What the pairs (s, t), s != t, of a tile give to the gates between them, the sum over its
// tokens s, in all lanes: decayed scores of the one product times the other's plain ones.
__device__ __forceinline__ float pairs16(const f32x4& p, const f32x4& z, int s0, int t0, int lane) {
  float x = 0.f;
#pragma unroll
  for (int r = 0; r < 4; ++r) x += s0 + 4 * (lane >> 4) + r != t0 + (lane & 15) ? p[r] * z[r] : 0.f;
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// One chunk, for a wave's 32 columns of a state of R rows, the scores being on their way into
// P.  Lane l % 32 is token t; the elements of o are columns c0 + held_row(r).
//   c = carry_t S^T q_t
//   o = c + sum over s of P[t][s] v_s
// and the state takes up the chunk.  REV: time runs back.  PAIR: c also takes what the
// state's rounding to bfloat16 leaves, and y_t . c is returned, with the rows y_t (the wave's
// 32 columns of them) in sy: what the tokens before the chunk give to the gates before t.
// The barrier behind which all waves' scores are in P comes after the state's products.
// Each step reads the next one's operands from LDS before it works on its own: the fences
// keep the compiler from reading them only where they are used.
template <typename Tin, int R, int C, bool REV, bool PAIR>
__device__ __forceinline__ float chunk_step(const Tin* sq, const Tin* sk, const Tin* sv, const Tin* sy,
                                            const Decays& dec, const Scores<Tin>& P, float scale, int c0,
                                            int lane, State<R / 32>& S, f32x16& o) {
  using F = typename Frag<Tin>::T;
  using TR = Tile<Tin, R>;
  using TC = Tile<Tin, C>;
  const int t = lane & 31;
  constexpr int K = R / 16, I = R / 32;
  F y[2], v[2];
  o = zero16();
  F q = TR::row_frag(sq, t, 0, lane);
#pragma unroll
  for (int kk = 0; kk < K; ++kk) {
    F qn = q;
    if (kk + 1 < K) qn = TR::row_frag(sq, t, kk + 1, lane);
    else v[0] = TC::col_frag(sv, c0, 0, lane);
    fence();
    const F s = state_frag<Tin>(S.s[kk >> 1], kk & 1);
    if constexpr (PAIR && sizeof(Tin) == 2) Frag<Tin>::mma(o, state_frag_low(S.s[kk >> 1], kk & 1, s), q);
    Frag<Tin>::mma(o, s, q);
    fence();
    q = qn;
  }
  const float carry = (REV ? dec.out[t] : dec.in[t] * scale) * S.f;
  if (S.decay(dec.total())) S.apply();
  const float inv = (REV ? scale : 1.f) * __builtin_amdgcn_rcpf(S.f);
  F k = TR::col_frag(sk, 0, 0, lane);
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    float w[8];
    weights8(REV ? dec.in : dec.out, kk, lane, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= inv;
    const Scaled<Tin> x(v[kk], w);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      F kn = k;
      if (i + 1 < I) kn = TR::col_frag(sk, 32 * (i + 1), kk, lane);
      else if (kk == 0) kn = TR::col_frag(sk, 0, 1, lane);
      if (kk == 0 && i == 0) v[1] = TC::col_frag(sv, c0, 1, lane);
      if constexpr (PAIR) {
        if (kk == 1 && i + 1 == I) {
          y[0] = TC::row_frag(sy + c0, t, 0, lane);
          y[1] = TC::row_frag(sy + c0, t, 1, lane);
        }
      }
      fence();
      x.mma_b(S.s[i], k);
      fence();
      k = kn;
    }
  }
  float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    o[r] *= carry;
    if constexpr (PAIR) dot[r & 3] += o[r] * (float)y[r >> 3][r & 7];
  }
  __syncthreads();
#pragma unroll
  for (int kk = 0; kk < 2; ++kk)
#pragma unroll
    for (int n = Scores<Tin>::TERMS - 1; n >= 0; --n)
      Frag<Tin>::mma(o, v[kk], P.frag(n, t, 16 * kk + 8 * (lane >> 5)));
  if constexpr (PAIR) {
    const float x = (dot[0] + dot[1]) + (dot[2] + dot[3]);
    return x + __shfl_xor(x, 32);
  }
  return 0.f;
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
// A chunk's outputs, lane l % 32 being a token: `chunk` is the address of its first row, the
// same for all threads; rows from `end` on do not exist, those from n on are zero.
template <typename Tout>
__device__ __forceinline__ void store_out(Tout* chunk, int64_t st, int c0, f32x16& o, int n, int end, int lane) {
  const int t = lane & 31;
  const uint32_t off = t * (uint32_t)st + c0 + 8 * (lane >> 5);
  if (n < kChunk) {
    if (t >= n) o = zero16();
    if (t >= end) return;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) store8(chunk + off + 16 * k, o, k);
}

}  // namespace dla
