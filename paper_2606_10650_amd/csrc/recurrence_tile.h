// What the recurrence's chunk kernels share: a chunk's tokens in LDS, its decays, and the
// states' 32 x 32 tiles.
//
// With a_t the sum of the chunk's log decays up to and with token t, a chunk of tokens
// turns the state S before it into outputs and the state behind it by
//   o_t = e^{a_t} S^T q_t + sum_{s <= t} e^{a_t - a_s} (q_t . k_s) v_s
//   S  <- e^{a_end} S + sum_s e^{a_end - a_s} k_s v_s^T
// so everything but the state's own decay is a matrix product.  Every factor is the decay
// between two points in time, taken from a difference: nothing is divided by a decay, and
// none overflows where the gates are not above zero.
#pragma once
#include "mfma.h"
#include "recurrence.h"

namespace dla {

// Tokens per chunk: 64 for bfloat16.  float32 operands have a sixteenth of the matrix
// rate, so the chunk's own products (32 tokens with each other) are kept small.
template <typename Tin>
constexpr int kChunk = sizeof(Tin) == 2 ? 64 : 32;

// CH rows of D values in LDS, in 16-byte pieces whose place in a row depends on the row,
// so that reads of one column by 16 rows, and of 64 (32: float32) bytes by the rows that
// one transposing read takes, spread over the banks.
template <typename Tin, int D>
struct Tile {
  static constexpr int CH = kChunk<Tin>;
  static constexpr int PE = 16 / (int)sizeof(Tin);   // elements per piece
  static constexpr int NP = D / PE;                  // pieces per row
  static constexpr int BYTES = CH * D * (int)sizeof(Tin);
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
  // operand with a column per lane and tokens 16 kk + 8 (lane / 32) + e: columns c0 +
  // lane % 32, or with PERM the columns in state_row's order.
  template <bool PERM>
  __device__ static __forceinline__ typename Frag<Tin>::T col_frag(const Tin* p, int c0, int kk,
                                                                   int lane) {
    const int g = lane >> 5;
    if constexpr (sizeof(Tin) == 2) {
      // a 16-lane group reads 4 rows of 16 columns, 8 bytes a lane, and lane i gets column i
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const int i = lane & 15, c4 = i & 3;
      const int col = c0 + (lane & 16) + (PERM ? 8 * (c4 & 1) + 4 * (c4 >> 1) : 4 * c4);
      const int row = 16 * kk + 8 * g + (i >> 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + at(row, col)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + at(row + 4, col)));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int m = lane & 31;
      const int col = c0 + (PERM ? (m & 16) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3) : m);
      f32x8 r;
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = p[at(16 * kk + 8 * g + e, col)];
      return r;
    }
  }
};

// Row of a state tile (or token of a score tile) that output element r of a lane half
// holds, when the tile's first operand gave lane m row perm_row(m): elements 8 kk .. 8 kk
// + 7 are then the 8 consecutive rows of a K = 16 step, and the tile serves as the next
// product's operand as it is.
__device__ __forceinline__ int perm_row(int m) {
  return (m & 16) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
}
__device__ __forceinline__ int held_row(int r, int lane) { return 16 * (r >> 3) + 8 * (lane >> 5) + (r & 7); }

// A chunk's tokens on their way from memory into a tile: loads are issued into registers
// and stored later.  Rows from `lim` on are zero, whatever memory holds there.
template <typename Tin, int D, int NT>
struct Stage {
  using TL = Tile<Tin, D>;
  static constexpr int N = TL::CH * TL::NP / NT;
  static_assert(TL::CH * TL::NP % NT == 0, "whole pieces per thread");
  u32x4 v[N];
  __device__ __forceinline__ void load(const Tin* base, int64_t st, int t0, int lim, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = i * NT + tid, row = x / TL::NP, pc = x % TL::NP, t = t0 + row;
      v[i] = u32x4{0u, 0u, 0u, 0u};
      if (t < lim) v[i] = *reinterpret_cast<const u32x4*>(base + t * st + pc * TL::PE);
    }
  }
  __device__ __forceinline__ void store(Tin* p, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = i * NT + tid, row = x / TL::NP, pc = x % TL::NP;
      *reinterpret_cast<u32x4*>(p + TL::at(row, pc * TL::PE)) = v[i];
    }
  }
};

// A chunk's decays in LDS.  In units of log2: a_t = hi + lo with hi whole, so that hi_t -
// hi_s is exact and the difference keeps float32's precision however large the sums are.
// A gate whose decay is below float32's smallest normal number (-inf among them) cuts:
// it counts as a step of -2^17 in hi, which no sum of a chunk's other gates reaches.
template <int CH>
struct Decays {
  float hi[CH], lo[CH];
  float in[CH];    // from before the chunk to token t: e^{a_t}
  float out[CH];   // from token t to the chunk's end: e^{a_end - a_t}
  float total;     // e^{a_end}
};

__device__ __forceinline__ float decay2(float hi_t, float lo_t, float hi_s, float lo_s) {
  return __builtin_amdgcn_exp2f((hi_t - hi_s) + (lo_t - lo_s));
}

constexpr float kCutGate = -87.33655f;   // ln of 2^-126

// By one wave: lane t holds the gate of token t.
template <int CH>
__device__ __forceinline__ void form_decays(Decays<CH>* d, float gate, int lane) {
  const bool cut = gate < kCutGate;
  double a = cut ? 0.0 : (double)gate * 1.4426950408889634;
  int n = cut ? 1 : 0;
#pragma unroll
  for (int o = 1; o < CH; o <<= 1) {
    const double x = __shfl_up(a, o);
    const int y = __shfl_up(n, o);
    if (lane >= o) {
      a += x;
      n += y;
    }
  }
  const double w = rint(a);
  const float hi = (float)w - 131072.f * (float)n, lo = (float)(a - w);
  const float eh = __shfl(hi, CH - 1), el = __shfl(lo, CH - 1);
  if (lane < CH) {
    d->hi[lane] = hi;
    d->lo[lane] = lo;
    d->in[lane] = decay2(hi, lo, 0.f, 0.f);
    d->out[lane] = decay2(eh, el, hi, lo);
    if (lane == CH - 1) d->total = decay2(hi, lo, 0.f, 0.f);
  }
}

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

// Eight of a chunk's per-token weights, from token 16 kk + 8 (lane / 32)
__device__ __forceinline__ void weights8(const float* w, int kk, int lane, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(w + 16 * kk + 8 * (lane >> 5));
  const float4 b = *reinterpret_cast<const float4*>(w + 16 * kk + 8 * (lane >> 5) + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// A state tile as a product's first operand (lane: column, elements: rows), rounded once
// to the inputs' type; with LOW also what that rounding left.
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

// A wave's columns c0 .. c0 + 31 of a state [R][C] (or of its transpose, stored [C][R]).
template <int NT_>
__device__ __forceinline__ void load_state(f32x16 (&s)[NT_], const float* p, int64_t rs, int64_t cs, int c0,
                                           int lane) {
#pragma unroll
  for (int i = 0; i < NT_; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      s[i][r] = p[(32 * i + held_row(r, lane)) * rs + (c0 + (lane & 31)) * cs];
}
template <int NT_>
__device__ __forceinline__ void store_state(const f32x16 (&s)[NT_], float* p, int64_t rs, int64_t cs, int c0,
                                            int lane) {
#pragma unroll
  for (int i = 0; i < NT_; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      p[(32 * i + held_row(r, lane)) * rs + (c0 + (lane & 31)) * cs] = s[i][r];
}

// Four consecutive values of an output row, rounded once to the output's type.
__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 x;
  x[0] = (__bf16)a; x[1] = (__bf16)b; x[2] = (__bf16)c; x[3] = (__bf16)d;
  *reinterpret_cast<bf16x4*>(p) = x;
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
// A 32 x 32 output tile: lane: token, elements: columns (out_row order)
template <typename Tout>
__device__ __forceinline__ void store_out(Tout* row, int c0, const f32x16& o, int lane) {
#pragma unroll
  for (int b = 0; b < 4; ++b)
    store4(row + c0 + 8 * b + 4 * (lane >> 5), o[4 * b], o[4 * b + 1], o[4 * b + 2], o[4 * b + 3]);
}

}  // namespace dla
