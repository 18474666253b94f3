// Root-mean-square norm of a residual stream: h = x + residual, y = w h / rms(h), with y in
// the inputs' type or in 8 bits with a scale per row; and its backward pass.
//
// A row lies in the registers of NT threads, NP pieces of 16 bytes each: one wave per row
// where that holds it (no LDS, no barrier) and rows are many, a workgroup otherwise.  Rows
// are read once and written once, so bytes bound the forward pass, and the backward pass
// but for dw: a workgroup goes over many rows with dw's sums of its columns in registers,
// leaves one partial sum per column, and a second kernel adds those up in a fixed order.
// 65536 rows of 2048 bfloat16: forward 204 us for 1.07 GB, 5.3 TB/s (a large copy 5.1),
// backward 208 us and 6 for dw; float32: 484 us, 4.4 TB/s, and 416, 5.2.  8192 rows of 16384
// float32: 484 us, 4.4 TB/s, and backward 476, 4.5, with seven registers a lane in scratch
// memory.  64 rows of 4096 to 8 bits: 6.8 us, most of it a launch.
// Rows may start at any element: a piece is read as it lies, whatever its alignment.
#include "dla_common.h"
#include "dla_train.h"
#include "piece.h"
#include "rms_norm.h"

namespace dla {
namespace {

// Eight-bit floating point (4 exponent, 3 mantissa bits, no infinity), round to nearest
// even; |x| <= 448 or NaN.
template <int N>
__device__ __forceinline__ void store_f8(uint8_t* p, int n, const float (&x)[N]) {
  struct __attribute__((packed, aligned(1))) Raw {
    uint32_t w[N / 4];
  } r;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    uint32_t u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
    r.w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], u, true);
  }
  if (n >= N) {
    *reinterpret_cast<Raw*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = (uint8_t)(r.w[i >> 2] >> (8 * (i & 3)));
  }
}

template <typename T>
__device__ __forceinline__ void load_weight(const NormArgs& a, int i, int n, float (&w)[Piece<T>::N]) {
  if (sizeof(T) == 4 || a.w_f32) {
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j) w[j] = j < n ? static_cast<const float*>(a.w)[i + j] : 0.f;
  } else {
    Piece<T>::load(static_cast<const T*>(a.w) + i, n, w);
  }
}

// A sum (or, with MAX, a maximum that lets a NaN through) over the NT threads of a row.
template <int NT, bool MAX>
__device__ __forceinline__ float over_row(float x, float* lds) {
  auto both = [](float p, float q) { return MAX ? (q > p || q != q ? q : p) : p + q; };
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = both(x, __shfl_xor(x, o));
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) x = both(x, lds[i]);
  }
  return x;
}

// A row whose largest |y| is below this, 448 times the smallest normal float32, is all zero
// in 8 bits: its scale would have fewer bits, and 448 / top no finite value.
constexpr float kLeastTop = 448.f * 0x1p-126f;

template <typename T, int NT, int NP, bool F8>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void norm_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N, PER = NT > 256 ? 1 : 256 / NT;
  __shared__ float lds[NT / 64];
  const int tid = threadIdx.x % NT;
  const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / NT;
  if (row >= a.rows) return;   // whole waves, and whole workgroups where they share a row
  float h[NP][N], w[NP][N], sum = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * NT + tid) * N, n = a.D - c;
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] = 0.f;
    if (n > 0) {
      Piece<T>::load(static_cast<const T*>(a.x.p) + row * a.x.st + c, n, h[i]);
      if (a.res.p) {
        float r[N];
        Piece<T>::load(static_cast<const T*>(a.res.p) + row * a.res.st + c, n, r);
#pragma unroll
        for (int j = 0; j < N; ++j) h[i][j] += r[j];
      }
      if constexpr (NT <= 256) load_weight<T>(a, c, n, w[i]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum += h[i][j] * h[i][j];
  }
  sum = over_row<NT, false>(sum, lds);
  float ms = sum / (float)a.D + a.eps, rstd = 1.f / sqrtf(ms);
  if (!(ms >= 0x1p-100f && ms <= 0x1.fffffep127f)) {
    // Squares that leave float32's range, in all threads of the row or in none: once more
    // with the row scaled by a power of two.  (An infinity or NaN in the row stays one.)
    const float f = ms < 1.f ? 0x1p100f : 0x1p-80f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) sum += (h[i][j] * f) * (h[i][j] * f);
    ms = over_row<NT, false>(sum, lds) / (float)a.D + a.eps * f * f;
    // below 2^-126 in root mean square, which eps = 0 or a subnormal one allows, r has no
    // finite value
    rstd = ms < 0x1p-52f ? 0.f : f / sqrtf(ms);
  }
  if (a.rstd && tid == 0) a.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * NT + tid) * N, n = a.D - c;
    if (n > 0) {
      if (a.h.p) Piece<T>::store(static_cast<T*>(a.h.p) + row * a.h.st + c, n, h[i]);
      // (1024 threads need 64 registers or fewer for two workgroups a compute unit)
      if constexpr (NT > 256) load_weight<T>(a, c, n, w[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        h[i][j] = h[i][j] * rstd * w[i][j];
        if constexpr (F8) {
          const float y = j < n ? fabsf(h[i][j]) : 0.f;
          top = y > top || y != y ? y : top;
        }
      }
      if constexpr (!F8) Piece<T>::store(static_cast<T*>(a.y.p) + row * a.y.st + c, n, h[i]);
    }
  }
  if constexpr (F8) {
    top = over_row<NT, true>(top, lds);
    if (tid == 0) a.y_scale[row] = top < kLeastTop ? 0.f : top / 448.f;
    const float inv = top < kLeastTop ? 0.f : 448.f / top;   // (a NaN stays one)
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = a.D - c;
      if (n > 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          // past 448 by rounding only
          const float y = h[i][j] * inv;
          h[i][j] = y > 448.f ? 448.f : (y < -448.f ? -448.f : y);
        }
        store_f8(static_cast<uint8_t*>(a.y.p) + row * a.y.st + c, n, h[i]);
      }
    }
  }
}

// dx = (dn - n mean(dn n)) / rms + dres with n = h / rms and dn = dy w; dw = sum of dy n.
// A row's pieces stay as they were loaded (half the registers of their values, and twice the
// waves that have loads under way); dy w and h / rms are formed where they are used.
template <typename T, int NT, int NP, bool WF32>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void norm_backward_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N, PER = NT > 256 ? 1 : 256 / NT;
  using Raw = typename Piece<T>::Raw;
  __shared__ float lds[NT / 64];
  __shared__ float sums[PER > 1 ? PER - 1 : 1][PER > 1 ? NT * N : 1];
  const int tid = threadIdx.x % NT, sub = threadIdx.x / NT;
  const int64_t step = (int64_t)gridDim.x * PER;
  Raw w[WF32 ? 1 : NP];
  float wf[WF32 ? NP : 1][N], dw[NP][N];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * NT + tid) * N, n = a.D - c;
#pragma unroll
    for (int j = 0; j < N; ++j) dw[i][j] = 0.f;
    if constexpr (WF32) {
#pragma unroll
      for (int j = 0; j < N; ++j) wf[i][j] = 0.f;
      if (n > 0) load_weight<T>(a, c, n, wf[i]);
    } else {
      w[i] = Piece<T>::raw(static_cast<const T*>(a.w) + c, n > 0 ? n : 0);
    }
  }
  auto weight = [&](int i, int j) {
    if constexpr (WF32) return wf[i][j];
    else return Piece<T>::value(w[i], j);
  };
  // a workgroup's waves that share a row end together
  for (int64_t row = (int64_t)blockIdx.x * PER + sub; row < a.rows; row += step) {
    const float rstd = a.rstd[row];
    Raw dy[NP], h[NP], r[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = a.D - c > 0 ? a.D - c : 0;
      dy[i] = Piece<T>::raw(static_cast<const T*>(a.y.p) + row * a.y.st + c, n);
      h[i] = Piece<T>::raw(static_cast<const T*>(a.h.p) + row * a.h.st + c, n);
      r[i] = Piece<T>::raw(static_cast<const T*>(a.res.p) + row * a.res.st + c, a.res.p ? n : 0);
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float x = Piece<T>::value(dy[i], j) * (Piece<T>::value(h[i], j) * rstd);
        dw[i][j] += x;
        sum += x * weight(i, j);
      }
    const float mean = over_row<NT, false>(sum, lds) / (float)a.D;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = a.D - c;
      float x[N];
#pragma unroll
      for (int j = 0; j < N; ++j)
        x[j] = Piece<T>::value(r[i], j) +
               (Piece<T>::value(dy[i], j) * weight(i, j) - Piece<T>::value(h[i], j) * rstd * mean) * rstd;
      if (n > 0) Piece<T>::store(static_cast<T*>(a.x.p) + row * a.x.st + c, n, x);
    }
  }
  if (!a.dw_part) return;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    // the workgroup's rows one after the other into one sum
    if constexpr (PER > 1) {
      __syncthreads();
      if (sub > 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) sums[sub - 1][j * NT + tid] = dw[i][j];
      }
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int k = 0; k < PER - 1; ++k)
#pragma unroll
          for (int j = 0; j < N; ++j) dw[i][j] += sums[k][j * NT + tid];
      }
    }
    const int c = (i * NT + tid) * N;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (sub == 0 && c + j < a.D) a.dw_part[(int64_t)blockIdx.x * a.D + c + j] = dw[i][j];
  }
}

// dw[c] = sum over the workgroups' parts: 32 columns a workgroup, 32 threads to a column,
// eight loads under way in each
__global__ __launch_bounds__(1024) void dw_kernel(const float* part, int parts, int D, float* dw) {
  __shared__ float sums[32][33];
  const int col = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
  float s = 0.f;
  if (c < D) {
    int i = r;
    for (; i + 224 < parts; i += 256) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = part[(int64_t)(i + 32 * j) * D + c];
      s += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    for (; i < parts; i += 32) s += part[(int64_t)i * D + c];
  }
  sums[r][col] = s;
  __syncthreads();
  if (r == 0 && c < D) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) x += sums[i][col];
    dw[c] = x;
  }
}

template <typename T, int NT, int NP>
hipError_t go(const NormArgs& a, int kind, hipStream_t st) {
  constexpr int PER = NT > 256 ? 1 : 256 / NT, BLOCK = NT > 256 ? NT : 256;
  const dim3 block(BLOCK);
  if (kind < 2) {
    // a launch has fewer than 2^32 threads
    constexpr int64_t most = 0xFFFFFFFFll / BLOCK * PER;
    NormArgs part = a;
    for (int64_t row = 0; row < a.rows; row += most) {
      part.rows = a.rows - row < most ? a.rows - row : most;
      part.x = a.x.from(row, sizeof(T));
      part.res = a.res.from(row, sizeof(T));
      part.h = a.h.from(row, sizeof(T));
      part.y = a.y.from(row, kind == 1 ? 1 : sizeof(T));
      part.rstd = a.rstd ? a.rstd + row : nullptr;
      part.y_scale = a.y_scale ? a.y_scale + row : nullptr;
      const dim3 grid((unsigned)((part.rows + PER - 1) / PER));
      if (kind == 0) hipLaunchKernelGGL((norm_kernel<T, NT, NP, false>), grid, block, 0, st, part);
      else hipLaunchKernelGGL((norm_kernel<T, NT, NP, true>), grid, block, 0, st, part);
    }
  } else if (sizeof(T) == 2 && !a.w_f32) hipLaunchKernelGGL((norm_backward_kernel<T, NT, NP, false>), dim3(a.groups), block, 0, st, a);
  else hipLaunchKernelGGL((norm_backward_kernel<T, NT, NP, true>), dim3(a.groups), block, 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t pick(const NormArgs& a, int kind, hipStream_t st) {
  const int pieces = (a.D + Piece<T>::N - 1) / Piece<T>::N;
  switch (norm_threads(a.rows, pieces)) {
    case 64:
      if (pieces <= 64) return go<T, 64, 1>(a, kind, st);
      if (pieces <= 128) return go<T, 64, 2>(a, kind, st);
      return go<T, 64, 4>(a, kind, st);
    case 256:
      if (pieces <= 256) return go<T, 256, 1>(a, kind, st);
      if (pieces <= 512) return go<T, 256, 2>(a, kind, st);
      if (pieces <= 1024) return go<T, 256, 4>(a, kind, st);
      return go<T, 256, 8>(a, kind, st);
    default:   // float32 rows of more than 8192 values
      if constexpr (sizeof(T) == 4) return go<T, 1024, 4>(a, kind, st);
      return hipErrorInvalidValue;
  }
}

}  // namespace

// Threads that share a row: a wave where it holds the row in 4 pieces a lane and there are
// rows enough to fill the chip, else 256, past 2048 pieces 1024.
int norm_threads(int64_t rows, int pieces) {
  if (pieces <= 64 || (pieces <= 256 && rows >= 1024)) return 64;
  return pieces <= 2048 ? 256 : 1024;
}

// Workgroups of the backward pass, each leaving one part of dw: four a compute unit, where
// there are rows for them.
int norm_groups(int64_t rows, int pieces) {
  const int nt = norm_threads(rows, pieces), per = nt > 256 ? 1 : 256 / nt;
  const int64_t groups = (rows + per - 1) / per;
  return (int)(groups < 1024 ? groups : 1024);
}

hipError_t launch_norm(const NormArgs& a, int dtype, int kind, hipStream_t st) {
  return dtype == DLA_BF16 ? pick<bf16_t>(a, kind, st) : pick<float>(a, kind, st);
}

hipError_t launch_norm_dw(const NormArgs& a, float* dw, hipStream_t st) {
  hipLaunchKernelGGL(dw_kernel, dim3((a.D + 31) / 32), dim3(1024), 0, st, a.dw_part, a.groups, a.D, dw);
  return hipGetLastError();
}

}  // namespace dla
