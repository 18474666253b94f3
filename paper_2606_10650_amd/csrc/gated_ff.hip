// The gated feed-forward block for a few rows, and what its products need around them: float32 or
// unaligned operands as planes of bfloat16, and the gradients of both projections' outputs.
#include "gated_ff.h"
#include "mfma.h"
#include "piece.h"

namespace dla {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

// A few rows: the weights are read once, 16 rows of each a workgroup, its waves taking K in turn; the rows of x
// are the products' columns, and come from the caches.  Bytes of the weights bound it: 2048 x 5504
// bfloat16, 45 MB, for one row 13 us, 3.5 TB/s, for 16 rows 16, for 64 27.  (By 64 K values in place of 32,
// whole lines: 16 and 18.)
template <typename T>
struct StepFrag {
  using F = typename Frag<T>::T;
  struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    F v;
  };
  // 8 values from k on, zero where they are not in front of K; the last are read from K - 8 on, so that
  // every load is whole
  __device__ __forceinline__ static F get(const T* row, int k, int K) {
    if (K >= 8) return reinterpret_cast<const Raw*>(row + (k + 8 <= K ? k : K - 8))->v;
    F r = Frag<T>::zero();
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < K) put(r, e, row[e]);
    return r;
  }
  __device__ __forceinline__ static void put(bf16x8& r, int e, bf16_t v) { r[e] = __builtin_bit_cast(__bf16, v.x); }
  __device__ __forceinline__ static void put(f32x8& r, int e, float v) { r[e] = v; }
  __device__ __forceinline__ static void shut(F& r, int k, int K) {
    const int first = k + 8 <= K ? k : K > 8 ? K - 8 : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (first + e < k) r[e] = 0;
  }
};
template <typename T, int NB>
__global__ __launch_bounds__(512) void ff_step_kernel(int rows, int D, int F, FfRows x, FfRows wg, FfRows wu, FfRows y,
                                                      FfRows g, FfRows u) {
  constexpr int WAVES = 8, KW = 32;    // K values a wave takes at a time
  using S = StepFrag<T>;
  __shared__ float sums[WAVES][2][NB][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t f = min((int64_t)blockIdx.x * 16 + l16, (int64_t)F - 1);   // (rows behind the last are not stored)
  const T* pg = static_cast<const T*>(wg.p) + f * wg.st;
  const T* pu = static_cast<const T*>(wu.p) + f * wu.st;
  const T* px[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) px[b] = static_cast<const T*>(x.p) + min(16 * b + l16, rows - 1) * x.st;
  f32x4 acc[2][NB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int k = wave * KW; k < D; k += WAVES * KW) {
    const int c = k + 8 * q;
    typename S::F a0 = S::get(pg, c, D), a1 = S::get(pu, c, D), v[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) v[b] = S::get(px[b], c, D);
    if (k + KW > D) {
      S::shut(a0, c, D);
      S::shut(a1, c, D);
#pragma unroll
      for (int b = 0; b < NB; ++b) S::shut(v[b], c, D);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      mma16(acc[0][b], a0, v[b]);
      mma16(acc[1][b], a1, v[b]);
    }
  }
  // the waves' sums in their order
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) sums[wave][i][b][l16][4 * q + r] = acc[i][b][r];
  __syncthreads();
  for (int e = threadIdx.x; e < NB * 256; e += 512) {
    const int b = e >> 8, m = (e >> 4) & 15, r = e & 15;
    const int64_t col = (int64_t)blockIdx.x * 16 + r, row = 16 * b + m;
    float gv = 0.f, uv = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      gv += sums[w][0][b][m][r];
      uv += sums[w][1][b][m][r];
    }
    if (row < rows && col < F) {
      const float v = gv * sigmoid(gv) * uv;
      if constexpr (sizeof(T) == 2) static_cast<__bf16*>(y.p)[row * y.st + col] = (__bf16)v;
      else static_cast<float*>(y.p)[row * y.st + col] = v;
      if (g.p) {
        static_cast<float*>(g.p)[row * g.st + col] = gv;
        static_cast<float*>(u.p)[row * u.st + col] = uv;
      }
    }
  }
}

// Three bfloat16 terms of a value, whose sum it is to float32's last digit.  A value that is not finite, or
// rounds to an infinity, is its first term: it makes every sum that it is in infinite or, by the other operand's
// terms of zero or other sign, NaN.
__device__ __forceinline__ void terms(float v, __bf16 (&t)[3]) {
  t[0] = (__bf16)v;
  float rest = v - (float)t[0];
  if (!(fabsf(rest) < __builtin_huge_valf())) rest = 0.f;
  t[1] = (__bf16)rest;
  t[2] = (__bf16)(rest - (float)t[1]);
}

// A piece of values to the planes.
template <typename T, int N>
__device__ __forceinline__ void put_planes(uint16_t* to, int64_t plane, const float (&v)[N]) {
  typedef __bf16 vec __attribute__((ext_vector_type(N)));
  if constexpr (sizeof(T) == 2) {
    vec r;
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = (__bf16)v[j];
    *reinterpret_cast<vec*>(to) = r;
  } else {
    vec r[3];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      __bf16 t[3];
      terms(v[j], t);
#pragma unroll
      for (int q = 0; q < 3; ++q) r[q][j] = t[q];
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<vec*>(to + q * plane) = r[q];
  }
}

template <typename T>
__global__ __launch_bounds__(256) void ff_pack_kernel(FfPacks sets) {
  constexpr int N = Piece<T>::N;
  const FfPack& p = sets.set[blockIdx.y];
  const int ld = (p.cols + 7) & ~7, per = ld / N;
  const int64_t total = p.rows * per, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const int64_t row = i / per;
    const int c = (int)(i % per) * N;
    float v[N];
    Piece<T>::load(static_cast<const T*>(p.from.p) + row * p.from.st + c, p.cols > c ? p.cols - c : 0, v);
    put_planes<T, N>(p.to + row * ld + c, p.rows * ld, v);
  }
}

// dg and du, formed in float32 and rounded once.  Of bfloat16 inputs they become bfloat16, which is what the matrix
// units multiply: an error of 2^-8 of each at most, that adds to the gradients' own rounding (16384 rows, 2048 to 5504:
// off by 0.0023 of the gradients' size against float64, of which rounding the results alone is 0.0017).  A second
// bfloat16 term of each gives 0.0017, by twice the products: forward and backward 3380 us in place of 2140.
template <typename T>
__global__ __launch_bounds__(256) void ff_parts_kernel(int64_t rows, int F, int ld, FfRows g, FfRows u, FfRows dy,
                                                       uint16_t* to) {
  constexpr int N = Piece<T>::N;
  const int per = ld / N;
  const int64_t total = rows * per, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const int64_t row = i / per;
    const int c = (int)(i % per) * N, n = F > c ? F - c : 0;
    float gv[N], uv[N], d[N], e[N];
#pragma unroll
    for (int h = 0; h < N; h += 4) {
      float x[4], y[4];
      const int left = n > h ? n - h : 0;
      Piece<float>::load(static_cast<const float*>(g.p) + row * g.st + c + h, left, x);
      Piece<float>::load(static_cast<const float*>(u.p) + row * u.st + c + h, left, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gv[h + j] = x[j];
        uv[h + j] = y[j];
      }
    }
    Piece<T>::load(static_cast<const T*>(dy.p) + row * dy.st + c, n, d);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float s = sigmoid(gv[j]);
      e[j] = d[j] * (gv[j] * s);
      d[j] = d[j] * uv[j] * (s * (1.f + gv[j] * (1.f - s)));
    }
    put_planes<T, N>(to + row * 2 * ld + c, rows * 2 * ld, d);
    put_planes<T, N>(to + (row * 2 + 1) * ld + c, rows * 2 * ld, e);
  }
}

unsigned groups_of(int64_t n) {
  const int64_t g = (n + 255) / 256;
  return (unsigned)(g < 65536 ? g : 65536);
}

template <typename T>
hipError_t step(int rows, int D, int F, FfRows x, FfRows wg, FfRows wu, FfRows y, FfRows g, FfRows u, hipStream_t st) {
  const dim3 grid((F + 15) / 16), block(512);
  switch ((rows + 15) / 16) {
    case 1: hipLaunchKernelGGL((ff_step_kernel<T, 1>), grid, block, 0, st, rows, D, F, x, wg, wu, y, g, u); break;
    case 2: hipLaunchKernelGGL((ff_step_kernel<T, 2>), grid, block, 0, st, rows, D, F, x, wg, wu, y, g, u); break;
    case 3: hipLaunchKernelGGL((ff_step_kernel<T, 3>), grid, block, 0, st, rows, D, F, x, wg, wu, y, g, u); break;
    default: hipLaunchKernelGGL((ff_step_kernel<T, 4>), grid, block, 0, st, rows, D, F, x, wg, wu, y, g, u); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ff_step(int64_t rows, int D, int F, int dtype, FfRows x, FfRows wg, FfRows wu, FfRows y, FfRows g,
                          FfRows u, hipStream_t st) {
  return dtype == DLA_BF16 ? step<bf16_t>((int)rows, D, F, x, wg, wu, y, g, u, st)
                           : step<float>((int)rows, D, F, x, wg, wu, y, g, u, st);
}

hipError_t launch_ff_pack(const FfPacks& sets, int dtype, hipStream_t st) {
  int64_t most = 0;
  for (const FfPack& p : sets.set) {
    const int64_t n = p.rows * (int64_t)(round_up(p.cols, 8) / (dtype == DLA_BF16 ? 8 : 4));
    if (n > most) most = n;
  }
  if (most == 0) return hipSuccess;
  const dim3 grid(groups_of(most), 3), block(256);
  if (dtype == DLA_BF16) hipLaunchKernelGGL(ff_pack_kernel<bf16_t>, grid, block, 0, st, sets);
  else hipLaunchKernelGGL(ff_pack_kernel<float>, grid, block, 0, st, sets);
  return hipGetLastError();
}

hipError_t launch_ff_parts(int64_t rows, int F, int dtype, FfRows g, FfRows u, FfRows dy, uint16_t* to, hipStream_t st) {
  const int ld = (int)round_up(F, 8), N = dtype == DLA_BF16 ? 8 : 4;
  const dim3 grid(groups_of(rows * (ld / N))), block(256);
  if (rows == 0) return hipSuccess;
  if (dtype == DLA_BF16) hipLaunchKernelGGL(ff_parts_kernel<bf16_t>, grid, block, 0, st, rows, F, ld, g, u, dy, to);
  else hipLaunchKernelGGL(ff_parts_kernel<float>, grid, block, 0, st, rows, F, ld, g, u, dy, to);
  return hipGetLastError();
}

}  // namespace dla
