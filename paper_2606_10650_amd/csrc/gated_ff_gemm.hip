// The products of the gated feed-forward block on the matrix units: bfloat16 operands, float32
// sums.  Tiles of the operands go through registers into LDS, two steps of K ahead, while the tiles
// before them are multiplied.
//
// A tile of rows whose K values are contiguous lies in LDS as kStep values a row, its 16-byte pieces
// exchanged by the row's number, so that sixteen lanes that read a piece of sixteen rows have all
// banks; a tile whose rows are K (an operand that is used transposed) as it lies in memory, 64-byte
// units exchanged by the row modulo 4, and is transposed by the reads of 4 rows of 16 columns.
// What lies outside an operand is zero.
//
// What bounds the products is the clock that the card's power allows (1.3 to 1.5 GHz on one card, at which the matrix
// units are busy for 59, 75 and 68% of the cycles, forward, dx and dW), then what a compute unit gets from its
// die's cache, some 20 bytes a clock.  16384 rows, 2048 to 5504, bfloat16: forward (both projections) 715 us, 1030 TFLOP/s, dx
// 610, 1210, both dW 695, 1060; a large library product reaches 1380, of these shapes 1085, 1144 and 738.  Copies
// straight from memory into LDS got in the way of its reads (dx 790 us); tiles asked for further ahead changed
// nothing; tiles' sums shared unevenly, so that every unit has the same work, lost the operands that
// neighbours share (dW 760).
#include <type_traits>

#include "gated_ff.h"
#include "mfma.h"

namespace dla {
namespace {

constexpr int kStep = 64;   // K values a step

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float silu(float z) {
  return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

// A tile of R rows (or columns) by kStep values of K in LDS.
template <int R, bool ALONG>   // ALONG: K values are contiguous
struct FfTile {
  static constexpr int BYTES = R * kStep * 2;
  static constexpr int PIECES = BYTES / 16;
  static constexpr int PR = kStep / 8;   // pieces of a row, where K is contiguous
  __device__ static __forceinline__ int swap(int row) { return (row / (16 / PR)) & (PR - 1); }
  // row and first column of the piece that lies at place p (ALONG: row, K value; else K value, column)
  __device__ static __forceinline__ int row(int p) { return ALONG ? p / PR : p / (R / 8); }
  __device__ static __forceinline__ int col(int p) {
    if (ALONG) return ((p % PR) ^ swap(p / PR)) * 8;
    const int k = p / (R / 8);
    return ((p % (R / 8)) ^ ((k & 3) << 2)) * 8;
  }
  // operand of a 32 x 32 x 16 product: row r0 + lane % 32, K values 16 kk + 8 (lane / 32) + e
  __device__ static __forceinline__ bf16x8 frag(const char* t, int r0, int kk, int lane) {
    if constexpr (ALONG) {
      const int r = r0 + (lane & 31), c = (2 * kk + (lane >> 5)) ^ swap(r);
      return *reinterpret_cast<const bf16x8*>(t + (r * PR + c) * 16);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 lds4;
      // 16 lanes read 4 rows of 16 columns, 8 bytes each, and lane i gets column i
      const int i = lane & 15, k = 16 * kk + 8 * (lane >> 5) + (i >> 2), c = r0 + (lane & 16) + 4 * (i & 3);
      const int byte = ((c * 2) ^ ((k & 3) << 6));
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(t + k * (R * 2) + byte));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(t + (k + 4) * (R * 2) + byte));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Where a thread's pieces of a tile come from: byte offsets from the tile's first element, or one
// that is outside.
constexpr uint32_t kOutside = 0x80000000u;

template <int R, bool ALONG, int THREADS>
struct FfLoad {
  using Tile = FfTile<R, ALONG>;
  static constexpr int N = Tile::PIECES / THREADS;
  static_assert(Tile::PIECES % THREADS == 0, "whole pieces per thread");
  uint32_t off[N];
  // `left`: rows (ALONG) or columns that the operand has from the tile's corner on; MIXED: 32 rows of
  // one operand and of another in turn
  template <bool MIXED>
  __device__ __forceinline__ void init(int64_t left, int64_t ld, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = i * THREADS + tid, c = Tile::col(p);
      int r = Tile::row(p);
      if (MIXED) r = (r >> 6) * 32 + (r & 31);
      off[i] = (ALONG ? r : c) < left ? (uint32_t)((r * ld + c) * 2) : kOutside;
    }
  }
  // Piece i of the step from `base` on, of which `left` K values are the operand's.
  __device__ __forceinline__ u32x4 get(int i, const uint16_t* base, int64_t left, int tid) const {
    const __amdgpu_buffer_rsrc_t src =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), (short)0, 0x7FFFFFFF, 0x00020000);
    uint32_t o = off[i];
    if (left < kStep) {
      const int p = i * THREADS + tid;
      if ((ALONG ? Tile::col(p) : Tile::row(p)) >= left) o = kOutside;
    }
    return __builtin_amdgcn_raw_buffer_load_b128(src, (int)o, 0, 0);
  }
};

// Row m and columns n .. n + 3 of a tile of C, where they are inside.
__device__ __forceinline__ void put4(const FfRows& r, int64_t m, int64_t n, int64_t N, int f32, const float (&v)[4]) {
  if (f32) {
    float* p = static_cast<float*>(r.p) + m * r.st + n;
    if (n + 4 <= N && ((uintptr_t)p & 15) == 0) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < N) p[e] = v[e];
  } else {
    __bf16* p = static_cast<__bf16*>(r.p) + m * r.st + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) p[e] = (__bf16)v[e];
  }
}

// A wave's place in a tile of C from its sums.  mine: kLine * 32 bytes of LDS.
constexpr int kLine = 144;

template <int KIND, int TM, int TN, int WM, int WN, bool F32>
__device__ __forceinline__ void ff_store(const FfGemm& p, const f32x16 (&acc)[TM / WM / 32][TN / WN / 32], int64_t m0,
                                         int64_t n0, char* mine, int lane, int wave) {
  constexpr int SM = TM / WM / 32, SN = TN / WN / 32, WIDTH = KIND == 0 ? TN / 2 : TN;
  const int wm = wave / WN, wn = wave % WN;
  const int64_t mw = m0 + wm * (TM / WM), nw = n0 + wn * (WIDTH / WN);   // the wave's corner
  const int l32 = lane & 31, half = lane >> 5;
  // A wave's columns of C, of one of the outputs, through LDS in rows of kLine bytes (so that eight lanes' pieces
  // have other banks), so that memory is written 16 bytes a lane.
  auto out = [&](auto kind, const FfRows& r, int64_t rows, int64_t m, int64_t c, auto value, auto for_later) {
    using T = decltype(kind);
    constexpr bool f32 = sizeof(T) == 4, later = decltype(for_later)::value;
    // value(e): element e of the lane; its row is m + l32, its columns c + out_row(e, lane); later: g and u,
    // which only the backward pass reads, are not to take the operands' place in the caches (with both in
    // bfloat16 675 us became 655); y, which the next product reads, may (float32, 8192 x 768 x 2048 with
    // that product behind it, 486 us, and 487 with y past the caches too)
    if (!r.p) return;
    const bool pieces = ((uintptr_t)r.p & 15) == 0 && r.st % (f32 ? 4 : 8) == 0;
    if (!pieces) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v[4] = {value(4 * e), value(4 * e + 1), value(4 * e + 2), value(4 * e + 3)};
        if ((uint64_t)(m + l32) < (uint64_t)rows) put4(r, m + l32, c + 8 * e + 4 * half, p.N, f32, v);
      }
      return;
    }
    {
      constexpr int N = 16 / (int)sizeof(T), PER = 32 / N;      // values of a piece, pieces of a row
      typedef T four __attribute__((ext_vector_type(4)));
      typedef T vec __attribute__((ext_vector_type(N)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        four v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (T)value(4 * e + q);
        *reinterpret_cast<four*>(mine + l32 * kLine + (8 * e + 4 * half) * (int)sizeof(T)) = v;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int t = 0; t < PER / 2; ++t) {
        const int row = (64 / PER) * t + lane / PER, col = N * (lane % PER);
        const vec v = *reinterpret_cast<const vec*>(mine + row * kLine + col * (int)sizeof(T));
        if ((uint64_t)(m + row) < (uint64_t)rows) {   // (m is below zero where a tile holds the end of one half)
          T* to = static_cast<T*>(r.p) + (m + row) * r.st + c + col;
          if (c + col + N <= p.N) {
            if (later) __builtin_nontemporal_store(v, reinterpret_cast<vec*>(to));
            else *reinterpret_cast<vec*>(to) = v;
          } else {
#pragma unroll
            for (int q = 0; q < N; ++q)
              if (c + col + q < p.N) to[q] = v[q];
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  };
  const typename std::conditional<F32, float, __bf16>::type type{};
  const std::false_type soon;
  const std::true_type later;
#pragma unroll
  for (int i = 0; i < SM; ++i) {
    const int64_t m = mw + 32 * i;
    if constexpr (KIND == 0) {
#pragma unroll
      for (int j = 0; j < SN; j += 2) {
        const int64_t c = nw + 16 * j;
        out(type, p.c, p.M, m, c, [&](int e) { return silu(acc[i][j][e]) * acc[i][j + 1][e]; }, soon);
        out(0.f, p.g, p.M, m, c, [&](int e) { return acc[i][j][e]; }, later);
        out(0.f, p.u, p.M, m, c, [&](int e) { return acc[i][j + 1][e]; }, later);
      }
    } else {
      // of kind 2 a tile's 32 rows may belong to both halves, where these are not multiples of 32 long
#pragma unroll
      for (int j = 0; j < SN; ++j) {
        auto value = [&](int e) { return acc[i][j][e]; };
        if constexpr (KIND == 1) {
          out(type, p.c, p.M, m, nw + 32 * j, value, soon);
        } else {
          if (m < p.half) out(type, p.c, p.rows, m, nw + 32 * j, value, soon);
          if (m + 32 > p.half) out(type, p.c2, p.rows, m - p.half, nw + 32 * j, value, soon);
        }
      }
    }
  }
}

// Where a tile lies in C: kGroup tiles of M go through the tiles of N together.
struct FfCorner {
  int64_t m, n;
};
constexpr int kGroup = 4;

template <int TM, int WIDTH>
__device__ __forceinline__ FfCorner corner_of(const FfPlan& w, int64_t tile) {
  const int64_t g0 = tile / ((int64_t)kGroup * w.tiles_n) * kGroup, in = tile - g0 * w.tiles_n;
  const int gm = (int)(w.tiles_m - g0 < kGroup ? w.tiles_m - g0 : kGroup);
  return FfCorner{(g0 + in % gm) * TM, (in / gm) * WIDTH};
}

// KIND as in gated_ff.h.  WM x WN waves, each with a tile of (TM / WM) x (TN / WN); of kind 0 the
// tile's columns are TN / 2 of B and as many of B2, 32 in turn, so that a wave has g and u of the
// same columns.
//
// The products' first operand is B's, so that a lane holds a row of C and four neighbours of its columns.
// A wave reads its operands of 16 K values ahead of the products of the 16 before; those of a step's
// first 16 follow the barrier that the step's last products are still to come behind, so that neither
// the barrier nor LDS makes the matrix unit wait.
template <int KIND, int TM, int TN, int WM, int WN, bool F32>
__global__ __launch_bounds__(64 * WM * WN) void ff_gemm_kernel(FfGemm p, FfPlan w) {
  constexpr int THREADS = 64 * WM * WN;
  constexpr bool AL = KIND != 2, BL = KIND == 0, MIXED = KIND == 0;
  using TA = FfTile<TM, AL>;
  using TB = FfTile<TN, BL>;
  constexpr int SM = TM / WM / 32, SN = TN / WN / 32, KK = kStep / 16;
  constexpr int WIDTH = KIND == 0 ? TN / 2 : TN;    // columns of C that a tile has
  constexpr int BUFFER = TA::BYTES + TB::BYTES;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;

  // workgroups that run together (every eighth on one die) have neighbouring tiles
  auto together = [](int64_t id, int64_t total) {
    const int64_t each = total / 8, rest = total % 8, x = id % 8;
    return x * each + (x < rest ? x : rest) + id / 8;
  };
  // a tile, or a part of the steps of one that is shared; those who have the same part of neighbouring
  // tiles run together, and find each other's operands in their die's cache
  int64_t tile, first = 0, last = w.steps;
  int part = 0;
  if (blockIdx.x < w.full) {
    tile = together(blockIdx.x, w.full);
  } else {
    const int64_t rest = w.tiles - w.full, id = together(blockIdx.x - w.full, rest * w.share);
    part = (int)(id / rest);
    tile = w.full + id % rest;
    first = w.begin(part);
    last = w.begin(part + 1);
  }
  const FfCorner corner = corner_of<TM, WIDTH>(w, tile);
  const int64_t m0 = corner.m, n0 = corner.n;

  FfLoad<TM, AL, THREADS> la;
  FfLoad<TN, BL, THREADS> lb;
  la.template init<false>(p.M - m0, p.lda, tid);
  lb.template init<MIXED>(p.N - n0, p.ldb, tid);

  const int64_t ksteps = w.steps / p.pairs;
  // where the next step to ask for lies
  const int64_t da = AL ? kStep : kStep * p.lda, db = BL ? kStep : kStep * p.ldb;
  int pair = 0;
  int64_t k = 0;
  const uint16_t *pa = nullptr, *pb = nullptr, *pb2 = nullptr;
  auto seek = [&]() {
    const int ia = (int)(p.ia >> (4 * pair)) & 15, ib = (int)(p.ib >> (4 * pair)) & 15;
    pa = p.a[ia] + (AL ? m0 * p.lda + k : k * p.lda + m0);
    pb = p.b[ib] + (BL ? n0 * p.ldb + k : k * p.ldb + n0);
    if (MIXED) pb2 = p.b2[ib] + n0 * p.ldb + k;
  };
  if (first < last) {
    pair = (int)(first / ksteps);
    k = (first - pair * ksteps) * kStep;
    seek();
  }
  constexpr int PIECES = la.N + lb.N;    // of a step, per thread
  int64_t todo = last - first;           // steps to ask for; those behind the last are zeros
  u32x4 piece[PIECES];
  auto get = [&](int i) {
    const int64_t left = todo > 0 ? p.K - k : 0;
    if (i < la.N) {
      piece[i] = la.get(i, pa, left, tid);
    } else {
      // (of kind 0 a wave's 64 pieces are of one operand)
      const int j = i - la.N;
      const bool second = MIXED && (((j * THREADS / 64 + wave) * (64 / TB::PR) >> 5) & 1);
      piece[i] = lb.get(j, second ? pb2 : pb, left, tid);
    }
  };
  auto put = [&](int i, int buf) {
    const int at = i < la.N ? i * THREADS * 16 : TA::BYTES + (i - la.N) * THREADS * 16;
    *reinterpret_cast<u32x4*>(smem + buf * BUFFER + at + tid * 16) = piece[i];
  };
  auto advance = [&]() {
    --todo;
    k += kStep;
    if (k < p.K) {
      pa += da;
      pb += db;
      if (MIXED) pb2 += db;
    } else if (todo > 0) {
      ++pair;
      k = 0;
      seek();
    }
  };

  f32x16 acc[SM][SN];
#pragma unroll
  for (int i = 0; i < SM; ++i)
#pragma unroll
    for (int j = 0; j < SN; ++j) acc[i][j] = zero16();
  bf16x8 fa[2][SM], fb[2][SN];
  auto read = [&](int buf, int kk, int to) {
    const char* a = smem + buf * BUFFER;
#pragma unroll
    for (int j = 0; j < SN; ++j) fb[to][j] = TB::frag(a + TA::BYTES, wn * (TN / WN) + 32 * j, kk, lane);
#pragma unroll
    for (int i = 0; i < SM; ++i) fa[to][i] = TA::frag(a, wm * (TM / WM) + 32 * i, kk, lane);
  };
  auto products = [&](int of, int i) {
#pragma unroll
    for (int j = 0; j < SN; ++j) Frag<bf16_t>::mma(acc[i][j], fb[of][j], fa[of][i]);
  };
  const int n = (int)(last - first);
  if (n > 0) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) get(i);
    advance();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) put(i, 0);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) get(i);
    advance();
    __syncthreads();
    read(0, 0, 0);
    for (int s = 0; s < n; ++s) {
      const int buf = s & 1;
      // Between the products the next step's pieces go from registers to LDS, and those of the step after
      // it are asked for.
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) {
          read(buf, kk + 1, (kk + 1) & 1);
        } else if (s + 1 < n) {
          __syncthreads();
          read(buf ^ 1, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < SM; ++i) {
          products(kk & 1, i);
          constexpr int ROWS = SM * (KK - 1);   // all before the barrier
          const int row = kk * SM + i;
          __builtin_amdgcn_sched_barrier(0);
          if (row < ROWS) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q)
              if (q * ROWS / PIECES == row) {
                put(q, buf ^ 1);
                get(q);
              }
            if (row == ROWS - 1) advance();
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
  }

  if (blockIdx.x < w.full) {
    __syncthreads();
    ff_store<KIND, TM, TN, WM, WN, F32>(p, acc, m0, n0, smem + wave * (32 * kLine), lane, wave);
  } else {
    // a part of a tile's sum, as the lanes hold it
    f32x4* to = reinterpret_cast<f32x4*>(p.part) + ((tile - w.full) * w.share + part) * (int64_t)(TM * TN / 4) + tid;
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
      for (int j = 0; j < SN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          to[((i * SN + j) * 4 + e) * THREADS] = f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
  }
}

// The tiles whose sums are in parts: these in their order, 32 rows of a wave's place in a workgroup of its own.
template <int KIND, int TM, int TN, int WM, int WN, bool F32>
__global__ __launch_bounds__(64) void ff_join_kernel(FfGemm p, FfPlan w) {
  constexpr int WAVES = WM * WN, SM = TM / WM / 32, SN = TN / WN / 32;
  __shared__ __align__(16) char smem[32 * kLine];
  const int lane = threadIdx.x, i = blockIdx.x % SM, wave = blockIdx.x / SM % WAVES;
  const int64_t tile = blockIdx.x / (SM * WAVES);
  const f32x4* part = reinterpret_cast<const f32x4*>(p.part) + tile * w.share * (int64_t)(TM * TN / 4) +
                      i * (SN * 4 * WAVES * 64) + wave * 64 + lane;
  f32x16 acc[1][SN];
#pragma unroll
  for (int j = 0; j < SN; ++j) acc[0][j] = zero16();
#pragma unroll 2
  for (int s = 0; s < w.share; ++s, part += TM * TN / 4) {
#pragma unroll
    for (int j = 0; j < SN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 v = part[(j * 4 + e) * (WAVES * 64)];
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[0][j][4 * e + q] += v[q];
      }
  }
  const FfCorner corner = corner_of<TM, KIND == 0 ? TN / 2 : TN>(w, w.full + tile);
  // (as if the tile were 32 rows a wave)
  const int64_t m0 = corner.m + wave / WN * (TM / WM - 32) + 32 * i;
  ff_store<KIND, 32 * WM, TN, WM, WN, F32>(p, acc, m0, corner.n, smem, lane, wave);
}

template <int KIND, int TM, int TN, int WM, int WN, bool F32>
hipError_t go(const FfGemm& p, const FfPlan& w, hipStream_t st) {
  constexpr size_t shm = 2 * (size_t)(TM + TN) * kStep * 2;
  static_assert(WM * WN * 32 * kLine <= shm, "a place for each wave");
  const auto k = ff_gemm_kernel<KIND, TM, TN, WM, WN, F32>;
  if (shm > 65536) {
    const hipError_t r = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)shm);
    if (r != hipSuccess) return r;
  }
  const int64_t rest = w.tiles - w.full;
  hipLaunchKernelGGL(k, dim3((unsigned)(w.full + rest * w.share)), dim3(64 * WM * WN), shm, st, p, w);
  if (rest) {
    const auto j = ff_join_kernel<KIND, TM, TN, WM, WN, F32>;
    hipLaunchKernelGGL(j, dim3((unsigned)(rest * WM * WN * (TM / WM / 32))), dim3(64), 0, st, p, w);
  }
  return hipGetLastError();
}

template <bool F32>
hipError_t pick(const FfGemm& p, const FfPlan& w, hipStream_t st) {
  if (w.large) {
    if (p.kind == 0) return go<0, 256, 256, 2, 4, F32>(p, w, st);
    if (p.kind == 1) return go<1, 256, 256, 2, 4, F32>(p, w, st);
    return go<2, 256, 256, 2, 4, F32>(p, w, st);
  }
  if (p.kind == 0) return go<0, 128, 128, 2, 2, F32>(p, w, st);
  if (p.kind == 1) return go<1, 128, 128, 2, 2, F32>(p, w, st);
  return go<2, 128, 128, 2, 2, F32>(p, w, st);
}

}  // namespace

FfPlan plan_ff_gemm(int kind, int64_t M, int64_t N, int64_t K, int pairs) {
  FfPlan best{};
  double least = 0;
  for (int large = 0; large < 2; ++large) {
    FfPlan w{};
    const int t = large ? 256 : 128, width = kind == 0 ? t / 2 : t;
    w.large = large;
    w.tiles_m = (int)((M + t - 1) / t);
    w.tiles_n = (int)((N + width - 1) / width);
    w.tiles = (int64_t)w.tiles_m * w.tiles_n;
    w.steps = (K > 0 ? (K + kStep - 1) / kStep : 1) * pairs;   // (without K one of zeros)
    // A step's time in microseconds; what a part costs to write and to read, and the joining.  A large tile has its
    // compute unit for itself.  Of small ones two share a unit, and those behind them follow without a pause, so
    // that more than two for each unit take a step's time each; one alone waits for its loads, and where some
    // units have two and others one the two set the time.  Of 8 sizes from 270 to 16384 rows, three products each,
    // tiles and shares by these are within 1.5% of the best of 13 tried on average, and within 10% (with up to two
    // workgroups a unit counted by their number 3.6% and 18%: 4130 x 1280 x 154 float32, forward, in 297 workgroups 67
    // us, in 396 57).
    const int64_t at_once = 256;
    const double step = large ? 1.7 : 0.62, part = large ? 0.12 : 0.03, join = 6.;
    const auto rounds = [&](int64_t n) {
      const double each = (double)n / at_once;
      if (large || n == 0) return (double)((n + at_once - 1) / at_once);
      return n <= at_once ? 1.25 : each < 1.8 ? 1.8 : each;
    };
    w.full = w.tiles / at_once * at_once;
    const int64_t rest = w.tiles - w.full;
    double time = (rounds(w.full) + rounds(rest)) * w.steps * step;
    int share = 1;
    for (int s = 2; rest && s <= 64 && s * 4 <= w.steps; ++s) {     // of 4 steps at least
      const double c = (rounds(w.full) * w.steps + rounds(rest * s) * ((w.steps + s - 1) / s)) * step + join + part * rest * s;
      if (c < time) {
        time = c;
        share = s;
      }
    }
    if (share > 1) w.share = share;
    else w.full = w.tiles;
    w.part_bytes = (size_t)(w.tiles - w.full) * w.share * t * t * 4;
    if (!large || time < least) {
      best = w;
      least = time;
    }
  }
  return best;
}

hipError_t launch_ff_gemm(const FfGemm& p, const FfPlan& w, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  // the plan is for as many pairs, each with whole steps: the kernel divides by the steps of one
  if (p.pairs < 1 || w.steps < p.pairs || w.steps % p.pairs) return hipErrorInvalidValue;
  return p.out_f32 ? pick<true>(p, w, st) : pick<false>(p, w, st);
}

}  // namespace dla
