// The products of the gated feed-forward block on the matrix units: bfloat16 operands, float32
// sums.  Tiles of the operands go from memory straight into LDS, two steps of K at a time, while
// the tiles before them are multiplied.
//
// A tile of rows whose K values are contiguous lies in LDS as 64 values a row, its 16-byte pieces
// exchanged by the row's number modulo 8, so that eight lanes that read a piece of eight rows
// have all banks; a tile whose rows are K (an operand that is used transposed) as it lies in
// memory, 64-byte units exchanged by the row modulo 4, and is transposed by the reads of 4 rows of
// 16 columns.  What lies outside an operand is zero.
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
  // row and first column of the piece that lies at place p (ALONG: row, K value; else K value, column)
  __device__ static __forceinline__ int row(int p) { return ALONG ? p >> 3 : p / (R / 8); }
  __device__ static __forceinline__ int col(int p) {
    if (ALONG) return ((p & 7) ^ ((p >> 3) & 7)) * 8;
    const int k = p / (R / 8);
    return ((p % (R / 8)) ^ ((k & 3) << 2)) * 8;
  }
  // operand of a 32 x 32 x 16 product: row r0 + lane % 32, K values 16 kk + 8 (lane / 32) + e
  __device__ static __forceinline__ bf16x8 frag(const char* t, int r0, int kk, int lane) {
    if constexpr (ALONG) {
      const int r = r0 + (lane & 31), c = (2 * kk + (lane >> 5)) ^ (r & 7);
      return *reinterpret_cast<const bf16x8*>(t + r * 128 + c * 16);
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
// that is outside.  `rows` and `cols` are what the operand has from the tile's corner on.
constexpr uint32_t kOutside = 0x80000000u;

template <int R, bool ALONG, int THREADS>
struct FfLoad {
  using Tile = FfTile<R, ALONG>;
  static constexpr int N = Tile::PIECES / THREADS;
  static_assert(Tile::PIECES % THREADS == 0, "whole pieces per thread");
  uint32_t off[N];
  // ALONG: the row is inside, whichever step; else the column
  __device__ __forceinline__ void init(int64_t left, int64_t ld, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = i * THREADS + tid, r = Tile::row(p), c = Tile::col(p);
      off[i] = (ALONG ? r : c) < left ? (uint32_t)((r * ld + c) * 2) : kOutside;
    }
  }
  // the step from `base` on, of which `left` K values are the operand's
  __device__ __forceinline__ void issue(const uint16_t* base, int64_t left, char* lds, int tid) const {
    const __amdgpu_buffer_rsrc_t src =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), (short)0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = i * THREADS + tid;
      const int k = ALONG ? Tile::col(p) : Tile::row(p);
      const uint32_t o = k < left ? off[i] : kOutside;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          src, (__attribute__((address_space(3))) void*)(lds + (i * THREADS + (tid & ~63)) * 16), 16, (int)o, 0, 0, 0);
    }
  }
};

__device__ __forceinline__ void put(const FfRows& r, int64_t row, int64_t col, float v, int f32) {
  if (f32) static_cast<float*>(r.p)[row * r.st + col] = v;
  else static_cast<__bf16*>(r.p)[row * r.st + col] = (__bf16)v;
}

// An element of C.
template <int KIND>
__device__ __forceinline__ void put_c(const FfGemm& p, int64_t m, int64_t n, float v) {
  if constexpr (KIND == 2) {
    const bool second = m >= p.half;
    const int64_t row = second ? m - p.half : m;
    const FfRows& r = second ? p.c2 : p.c;
    if (row < p.rows && r.p) put(r, row, n, v, p.out_f32);
  } else {
    put(p.c, m, n, v, p.out_f32);
  }
}

// KIND as in gated_ff.h.  WM x WN waves, each with a tile of (TM / WM) x (TN / WN); of kind 0 the
// tile's columns are TN / 2 of B and as many of B2, 32 in turn, so that a wave has g and u of the
// same columns.
template <int KIND, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void ff_gemm_kernel(FfGemm p, int tiles_m, int tiles_n) {
  constexpr int THREADS = 64 * WM * WN;
  constexpr bool AL = KIND != 2, BL = KIND == 0;
  using TA = FfTile<TM, AL>;
  using TB = FfTile<TN, BL>;
  constexpr int SM = TM / WM / 32, SN = TN / WN / 32;
  constexpr int WIDTH = KIND == 0 ? TN / 2 : TN;    // columns of C that a tile has
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;

  // workgroups that run together (every eighth on one die) have neighbouring tiles
  const int64_t total = (int64_t)tiles_m * tiles_n * p.split;
  int64_t id = blockIdx.x;
  {
    const int64_t each = total / 8, rest = total % 8, x = id % 8, y = id / 8;
    id = x * each + (x < rest ? x : rest) + y;
  }
  const int64_t tiles = (int64_t)tiles_m * tiles_n;
  const int part = (int)(id / tiles);
  id %= tiles;
  constexpr int GROUP = 8;   // tiles of M that go through the tiles of N together
  const int64_t g0 = id / ((int64_t)GROUP * tiles_n) * GROUP;
  const int gm = (int)(tiles_m - g0 < GROUP ? tiles_m - g0 : GROUP);
  const int64_t in = id - g0 * tiles_n;
  const int64_t m0 = (g0 + in % gm) * TM, n0 = (in / gm) * WIDTH;

  FfLoad<TM, AL, THREADS> la;
  FfLoad<TN, BL, THREADS> lb;
  la.init(p.M - m0, p.lda, tid);
  if constexpr (KIND == 0) {
    // rows 64 i .. 64 i + 31 of the tile are B's 32 i .., the next 32 B2's
#pragma unroll
    for (int i = 0; i < lb.N; ++i) {
      const int q = i * THREADS + tid, r = TB::row(q), n = (r >> 6) * 32 + (r & 31);
      lb.off[i] = n < p.N - n0 ? (uint32_t)((n * p.ldb + TB::col(q)) * 2) : kOutside;
    }
  } else {
    lb.init(p.N - n0, p.ldb, tid);
  }

  const int64_t ksteps = (p.K + kStep - 1) / kStep, steps = ksteps * p.pairs;
  const int64_t first = steps * part / p.split, last = steps * (part + 1) / p.split;

  auto issue = [&](int64_t s, int buf) {
    const int pair = (int)(s / ksteps);
    const int64_t k0 = (s % ksteps) * kStep;
    char* at = smem + buf * (TA::BYTES + TB::BYTES);
    const uint16_t* a = p.a[p.ia[pair]];
    la.issue(AL ? a + m0 * p.lda + k0 : a + k0 * p.lda + m0, p.K - k0, at, tid);
    const uint16_t* b = p.b[p.ib[pair]];
    if constexpr (KIND == 0) {
      const uint16_t* b2 = p.b2[p.ib[pair]];
      const __amdgpu_buffer_rsrc_t s1 = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(b + n0 * p.ldb + k0), (short)0, 0x7FFFFFFF, 0x00020000);
      const __amdgpu_buffer_rsrc_t s2 = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(b2 + n0 * p.ldb + k0), (short)0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
      for (int i = 0; i < lb.N; ++i) {
        // a wave's 64 pieces are 8 rows, all of one operand
        const int q = i * THREADS + tid;
        const uint32_t o = TB::col(q) < p.K - k0 ? lb.off[i] : kOutside;
        auto* to = (__attribute__((address_space(3))) void*)(at + TA::BYTES + (i * THREADS + (tid & ~63)) * 16);
        if (((i * THREADS / 64 + wave) >> 2) & 1)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(s2, to, 16, (int)o, 0, 0, 0);
        else
          __builtin_amdgcn_raw_ptr_buffer_load_lds(s1, to, 16, (int)o, 0, 0, 0);
      }
    } else {
      lb.issue(BL ? b + n0 * p.ldb + k0 : b + k0 * p.ldb + n0, p.K - k0, at + TA::BYTES, tid);
    }
  };

  f32x16 acc[SM][SN];
#pragma unroll
  for (int i = 0; i < SM; ++i)
#pragma unroll
    for (int j = 0; j < SN; ++j) acc[i][j] = zero16();
  if (first < last) issue(first, 0);
  for (int64_t s = first; s < last; ++s) {
    const int buf = (int)(s - first) & 1;
    // this step's tiles have come, the other's are no longer read
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // vmcnt 0
    __syncthreads();
    if (s + 1 < last) issue(s + 1, buf ^ 1);
    const char* a = smem + buf * (TA::BYTES + TB::BYTES);
    const char* b = a + TA::BYTES;
#pragma unroll
    for (int kk = 0; kk < kStep / 16; ++kk) {
      bf16x8 fa[SM], fb[SN];
#pragma unroll
      for (int i = 0; i < SM; ++i) fa[i] = TA::frag(a, wm * (TM / WM) + 32 * i, kk, lane);
#pragma unroll
      for (int j = 0; j < SN; ++j) fb[j] = TB::frag(b, wn * (TN / WN) + 32 * j, kk, lane);
#pragma unroll
      for (int i = 0; i < SM; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) Frag<bf16_t>::mma(acc[i][j], fa[i], fb[j]);
    }
  }

  const int l32 = lane & 31;
#pragma unroll
  for (int i = 0; i < SM; ++i) {
    if constexpr (KIND == 0) {
#pragma unroll
      for (int j = 0; j < SN; j += 2) {
        const int64_t n = n0 + (wn * (TN / WN) + 32 * j) / 2 + l32;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t m = m0 + wm * (TM / WM) + 32 * i + out_row(e, lane);
          if (m < p.M && n < p.N) {
            const float g = acc[i][j][e], u = acc[i][j + 1][e];
            put(p.c, m, n, silu(g) * u, p.out_f32);
            if (p.g.p) {
              put(p.g, m, n, g, p.out_f32);
              put(p.u, m, n, u, p.out_f32);
            }
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < SN; ++j) {
        const int64_t n = n0 + wn * (TN / WN) + 32 * j + l32;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t m = m0 + wm * (TM / WM) + 32 * i + out_row(e, lane);
          if (m < p.M && n < p.N) {
            if (p.split > 1) p.part[((int64_t)part * p.M + m) * p.N + n] = acc[i][j][e];
            else put_c<KIND>(p, m, n, acc[i][j][e]);
          }
        }
      }
    }
  }
}

// C = the sum of the parts, in their order
template <int KIND>
__global__ __launch_bounds__(256) void ff_sum_kernel(FfGemm p) {
  const int64_t n = p.M * p.N, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    float s = 0.f;
    for (int k = 0; k < p.split; ++k) s += p.part[k * n + i];
    put_c<KIND>(p, i / p.N, i % p.N, s);
  }
}

template <int KIND, int TM, int TN, int WM, int WN>
hipError_t go(const FfGemm& p, hipStream_t st) {
  constexpr int WIDTH = KIND == 0 ? TN / 2 : TN;
  const int64_t tm = (p.M + TM - 1) / TM, tn = (p.N + WIDTH - 1) / WIDTH;
  const size_t shm = 2 * (size_t)(TM + TN) * kStep * 2;
  const auto k = ff_gemm_kernel<KIND, TM, TN, WM, WN>;
  if (shm > 65536) {
    const hipError_t r = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)shm);
    if (r != hipSuccess) return r;
  }
  hipLaunchKernelGGL(k, dim3((unsigned)(tm * tn * p.split)), dim3(64 * WM * WN), shm, st, p, (int)tm, (int)tn);
  return hipGetLastError();
}

bool large(int kind, int64_t M, int64_t N) {
  const int64_t width = kind == 0 ? 128 : 256;
  return ((M + 255) / 256) * ((N + width - 1) / width) >= 192;
}

}  // namespace

// Parts of the sum over K: as many as still give every compute unit a tile, of at least 8 steps.
int ff_split(int kind, int64_t M, int64_t N, int64_t K, int pairs) {
  if (kind == 0 || M == 0 || large(kind, M, N)) return 1;
  const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128), steps = (K + kStep - 1) / kStep * pairs;
  int64_t s = 512 / tiles;
  if (s > steps / 8) s = steps / 8;
  if (s > 16) s = 16;
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_ff_gemm(const FfGemm& p, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  hipError_t r;
  if (large(p.kind, p.M, p.N)) {
    if (p.kind == 0) r = go<0, 256, 256, 2, 4>(p, st);
    else if (p.kind == 1) r = go<1, 256, 256, 2, 4>(p, st);
    else r = go<2, 256, 256, 2, 4>(p, st);
  } else {
    if (p.kind == 0) r = go<0, 128, 128, 2, 2>(p, st);
    else if (p.kind == 1) r = go<1, 128, 128, 2, 2>(p, st);
    else r = go<2, 128, 128, 2, 2>(p, st);
  }
  if (r == hipSuccess && p.split > 1) {
    const int64_t groups = (p.M * p.N + 255) / 256;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536)), block(256);
    if (p.kind == 1) hipLaunchKernelGGL(ff_sum_kernel<1>, grid, block, 0, st, p);
    else hipLaunchKernelGGL(ff_sum_kernel<2>, grid, block, 0, st, p);
    r = hipGetLastError();
  }
  return r;
}

}  // namespace dla
