// The norm behind a block with its gate, the scaled residual sum, and the norm before the next
// block:  n = r x w, b = n silu(z), h = res + scale b, y = r' h w'; and its backward pass.
//
// A group of D values lies in the registers of NT threads, NP pieces of 16 bytes each: as few
// lanes of a wave as hold a head (128 bfloat16 values: 16), a wave for a row where rows are many, a
// workgroup otherwise.  Everything is read once and written once, so bytes bound both passes, and
// the backward pass but for the weights' gradients: a thread stays at its columns of its group
// and goes along the rows with their sums in registers; a workgroup leaves one part of each, and
// a second kernel adds the parts in a fixed order.  h is not read back in the backward pass but
// formed again from x, gate and residual, so that nothing depends on how h was rounded.
//
// 65536 rows of 16 heads of 128 bfloat16 values with gate, forward 0.8 GB in 165 us, 4.9 TB/s, backward 1.3 GB in
// 258, 5.2; 16384 rows of 2048 with residual and next norm, 0.27 GB in 61, 4.4, and 0.4 GB in 94, 4.3.  64 such rows
// take 5.4 us, nearly all of it waiting for two loads and two sums.
#include "gated_norm.h"
#include "piece.h"

namespace dla {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

// The sum over the NT threads of a group, in a fixed order.
template <int NT>
__device__ __forceinline__ float over_group(float x, float* lds) {
#pragma unroll
  for (int o = 1; o < (NT < 64 ? NT : 64); o <<= 1) x += __shfl_xor(x, o);
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    const float* mine = lds + threadIdx.x / NT * (NT / 64);
    x = mine[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) x += mine[i];
  }
  return x;
}

// 1 / sqrt(mean(v^2) + eps)
template <int NT, int NP, int N>
__device__ __forceinline__ float rstd_of(const float (&v)[NP][N], int D, float eps, float* lds) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) sum += v[i][j] * v[i][j];
  sum = over_group<NT>(sum, lds);
  float ms = sum / (float)D + eps, rstd = 1.f / sqrtf(ms);
  const bool out = !(ms >= 0x1p-100f && ms <= 0x1.fffffep127f);
  // Squares that leave float32's range (in all threads of the group or in none; where a wave or a
  // workgroup holds several groups all of them take part): once more with the values scaled by a power of
  // two.  An infinity or NaN stays one.
  if (NT < 64 ? __any(out) : NT == 128 ? __syncthreads_or(out) : out) {
    const float f = ms < 1.f ? 0x1p100f : 0x1p-80f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) sum += (v[i][j] * f) * (v[i][j] * f);
    ms = over_group<NT>(sum, lds) / (float)D + eps * f * f;
    if (out) rstd = ms < 0x1p-52f ? 0.f : f / sqrtf(ms);
  }
  return rstd;
}

// Where a thread works: its group, and the rows row0, row0 + step, ...
template <int NT>
struct Place {
  static constexpr int PER = NT > 256 ? 1 : 256 / NT;   // groups a workgroup has at a time
  int g, sub;
  int64_t row0, step;
  bool any;
  __device__ __forceinline__ explicit Place(const GatedNormArgs& a) {
    const int side = a.G < PER ? a.G : PER, along = PER / side;   // groups side by side, rows
    sub = threadIdx.x / NT;
    g = (int)(blockIdx.x % a.gcols) * PER + sub % side;
    row0 = (int64_t)(blockIdx.x / a.gcols) * along + sub / side;
    step = a.groups * along;
    any = sub < side * along && g < a.G;
  }
};

template <typename T>
__device__ __forceinline__ const T* at(const GroupRows& r, int64_t row, int g) {
  return static_cast<const T*>(r.p) + row * r.st + g * r.sg;
}
template <typename T>
__device__ __forceinline__ T* out(const GroupRows& r, int64_t row, int g) {
  return static_cast<T*>(r.p) + row * r.st + g * r.sg;
}

template <typename T, int NT, int NP>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void gated_norm_kernel(GatedNormArgs a) {
  constexpr int N = Piece<T>::N;
  using Raw = typename Piece<T>::Raw;
  __shared__ float lds[(NT > 256 ? NT : 256) / 64];
  const Place<NT> p(a);
  const int tid = threadIdx.x % NT;
  // all lanes of a wave go round together: those without a row or group hold zeros
  for (int64_t base = p.row0 - p.sub / (a.G < p.PER ? a.G : p.PER); base < a.rows; base += p.step) {
    const int64_t row = p.row0 + (base - (p.row0 - p.sub / (a.G < p.PER ? a.G : p.PER)));
    const bool any = p.any && row < a.rows;
    float v[NP][N];
    Raw z[NP], res[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
      const Raw x = Piece<T>::raw(at<T>(a.x, row, p.g) + c, n);
      z[i] = Piece<T>::raw(at<T>(a.gate, row, p.g) + c, a.gate.p ? n : 0);
      res[i] = Piece<T>::raw(at<T>(a.res, row, p.g) + c, a.res.p ? n : 0);
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = Piece<T>::value(x, j);
    }
    float r = rstd_of<NT, NP, N>(v, a.D, a.eps, lds);
    if (a.rstd && any && tid == 0) a.rstd[row * a.G + p.g] = r;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
      float w[N];
      load_floats<T>(a.w, a.w_f32, (int64_t)(a.per_group ? p.g : 0) * a.D + c, n, w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[i][j] = v[i][j] * r * w[j];
        if (a.gate.p) {
          const float zj = Piece<T>::value(z[i], j);
          v[i][j] *= zj * sigmoid(zj);
        }
        v[i][j] = a.scale * v[i][j] + Piece<T>::value(res[i], j);
      }
      if (n > 0) Piece<T>::store(out<T>(a.h, row, p.g) + c, n, v[i]);
    }
    if (!a.w2) continue;
    r = rstd_of<NT, NP, N>(v, a.D, a.eps, lds);
    if (a.rstd2 && any && tid == 0) a.rstd2[row] = r;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
      float w[N];
      load_floats<T>(a.w2, a.w_f32, c, n, w);
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = v[i][j] * r * w[j];
      if (n > 0) Piece<T>::store(out<T>(a.y, row, p.g) + c, n, v[i]);
    }
  }
}

// A workgroup's sums of the same columns into one, in a fixed order: those of the subs `stride`
// apart into the first `stride`.
template <int NT, int N, int PER>
__device__ __forceinline__ void gather(float (&s)[N], int sub, int stride, int subs, float* lds) {
  if constexpr (PER > 1) {
    const int tid = threadIdx.x % NT;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) lds[(j * PER + sub) * NT + tid] = s[j];
    __syncthreads();
    if (sub < stride)
      for (int k = sub + stride; k < subs; k += stride)
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] += lds[(j * PER + k) * NT + tid];
  }
}

// Waves a SIMD of the backward pass.  With gate and next norm a thread of 8 values needs more than a fourth of the
// registers (65536 x 2048 bfloat16: within a fourth 683 us, within a third 457).  Workgroups of 512 and 1024 threads
// keep to a fourth, and those of 8 values a thread with gate and next norm, or with more than one piece a thread, keep
// some values in memory (100 to 416 bytes a thread): 16384 x 4096 bfloat16 with gate, residual and next norm 366 us, 2.9
// TB/s, without gate 176, 4.6; 4096 x 16384 bfloat16 672 and float32 1103, 1.6 and 2.0.
template <typename T>
__host__ __device__ constexpr int waves_of(int nt, bool both) {
  return sizeof(T) == 2 && both && nt <= 256 ? 3 : 4;
}

template <typename T, int NT, int NP, bool GATE, bool NEXT>
__global__ __launch_bounds__(NT > 256 ? NT : 256, waves_of<T>(NT, GATE && NEXT)) void gated_norm_backward_kernel(GatedNormArgs a) {
  constexpr int N = Piece<T>::N, PER = Place<NT>::PER;
  using Raw = typename Piece<T>::Raw;
  __shared__ float lds[(NT > 256 ? NT : 256) / 64];
  __shared__ float sums[PER > 1 ? PER * NT * N : 1];
  const Place<NT> p(a);
  const int tid = threadIdx.x % NT, side = a.G < PER ? a.G : PER, along = PER / side;
  float dw[NP][N], dw2[NP][N];
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) dw[i][j] = dw2[i][j] = 0.f;
  const int64_t first = p.row0 - p.sub / side;
  for (int64_t base = first; base < a.rows; base += p.step) {
    const int64_t row = p.row0 + (base - first);
    const bool any = p.any && row < a.rows;
    const float r = any ? a.rstd[row * a.G + p.g] : 0.f;
    Raw x[NP], z[NP], d[NP];
    float dh[NP][N];
    float w2sum = 0.f, r2 = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
      x[i] = Piece<T>::raw(at<T>(a.x, row, p.g) + c, n);
      z[i] = Piece<T>::raw(at<T>(a.gate, row, p.g) + c, GATE ? n : 0);
      const Raw q = Piece<T>::raw(at<T>(a.h, row, p.g) + c, a.h.p ? n : 0);
#pragma unroll
      for (int j = 0; j < N; ++j) dh[i][j] = Piece<T>::value(q, j);
    }
    if constexpr (NEXT) {
      // through the next norm: dh += r' (dy w' - n' mean(dy w' n'))
      r2 = any ? a.rstd2[row] : 0.f;
      float h[NP][N];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
        d[i] = Piece<T>::raw(at<T>(a.y, row, p.g) + c, n);
        const Raw q = Piece<T>::raw(at<T>(a.res, row, p.g) + c, a.res.p ? n : 0);
        float w[N], w2[N];
        load_floats<T>(a.w, a.w_f32, (int64_t)(a.per_group ? p.g : 0) * a.D + c, n, w);
        load_floats<T>(a.w2, a.w_f32, c, n, w2);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float b = Piece<T>::value(x[i], j) * r * w[j];
          if constexpr (GATE) {
            const float zj = Piece<T>::value(z[i], j);
            b *= zj * sigmoid(zj);
          }
          h[i][j] = (a.scale * b + Piece<T>::value(q, j)) * r2;
          const float t = Piece<T>::value(d[i], j) * h[i][j];
          dw2[i][j] += t;
          w2sum += t * w2[j];
        }
      }
      const float mean = over_group<NT>(w2sum, lds) / (float)a.D;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
        float w2[N];
        load_floats<T>(a.w2, a.w_f32, c, n, w2);
#pragma unroll
        for (int j = 0; j < N; ++j) dh[i][j] += r2 * (Piece<T>::value(d[i], j) * w2[j] - h[i][j] * mean);
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
      if (n > 0 && a.dres.p) Piece<T>::store(out<T>(a.dres, row, p.g) + c, n, dh[i]);
      float w[N], dz[N];
      load_floats<T>(a.w, a.w_f32, (int64_t)(a.per_group ? p.g : 0) * a.D + c, n, w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float nx = Piece<T>::value(x[i], j) * r;
        float db = a.scale * dh[i][j];
        if constexpr (GATE) {
          const float zj = Piece<T>::value(z[i], j), s = sigmoid(zj);
          dz[j] = db * nx * w[j] * (s * (1.f + zj * (1.f - s)));
          db *= zj * s;
        }
        dw[i][j] += db * nx;
        dh[i][j] = db * w[j];     // the gradient of n
        sum += dh[i][j] * nx;
      }
      if (GATE && n > 0 && a.dgate.p) Piece<T>::store(out<T>(a.dgate, row, p.g) + c, n, dz);
    }
    const float mean = over_group<NT>(sum, lds) / (float)a.D;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * NT + tid) * N, n = any && a.D > c ? a.D - c : 0;
#pragma unroll
      for (int j = 0; j < N; ++j) dh[i][j] = r * (dh[i][j] - Piece<T>::value(x[i], j) * r * mean);
      if (n > 0) Piece<T>::store(out<T>(a.dx, row, p.g) + c, n, dh[i]);
    }
  }
  const int64_t line = blockIdx.x / a.gcols;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * NT + tid) * N;
    if (a.dw_part) {
      // per group: subs of the same group; shared: all
      gather<NT, N, PER>(dw[i], p.sub, a.per_group ? side : 1, side * along, sums);
      if (a.per_group) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (p.sub < side && p.g < a.G && c + j < a.D) a.dw_part[(line * a.G + p.g) * a.D + c + j] = dw[i][j];
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (p.sub == 0 && c + j < a.D) a.dw_part[(int64_t)blockIdx.x * a.D + c + j] = dw[i][j];
      }
    }
    if (NEXT && a.dw2_part) {
      gather<NT, N, PER>(dw2[i], p.sub, 1, side * along, sums);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (p.sub == 0 && c + j < a.D) a.dw2_part[(int64_t)blockIdx.x * a.D + c + j] = dw2[i][j];
    }
  }
}

// dw[c] = the sum of the parts' column c, of up to two weights: 32 columns a workgroup, 32 threads to a column,
// in a fixed order, in float64
struct PartSum {
  const float* part;
  int64_t parts, width;
  float* dw;
};
__global__ __launch_bounds__(1024) void part_sum_kernel(PartSum p0, PartSum p1, unsigned blocks0) {
  __shared__ double sums[32][33];
  const bool second = blockIdx.x >= blocks0;
  const float* part = second ? p1.part : p0.part;
  const int64_t parts = second ? p1.parts : p0.parts, width = second ? p1.width : p0.width;
  const int col = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t c = (int64_t)(second ? blockIdx.x - blocks0 : blockIdx.x) * 32 + col;
  double s = 0.;
  if (c < width) {
    int64_t i = r;
    for (; i + 96 < parts; i += 128) {
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = part[(i + 32 * j) * width + c];
      s += ((double)x[0] + x[1]) + ((double)x[2] + x[3]);
    }
    for (; i < parts; i += 32) s += part[i * width + c];
  }
  sums[r][col] = s;
  __syncthreads();
  if (r == 0 && c < width) {
    for (int i = 1; i < 32; ++i) s += sums[i][col];
    (second ? p1.dw : p0.dw)[c] = (float)s;
  }
}

template <typename T, int NT, int NP>
hipError_t forward(const GatedNormArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.groups * a.gcols)), block(NT > 256 ? NT : 256);
  hipLaunchKernelGGL((gated_norm_kernel<T, NT, NP>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T, int NT, int NP>
hipError_t backward(const GatedNormArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.groups * a.gcols)), block(NT > 256 ? NT : 256);
  if (a.w2 && a.y.p) {
    if (a.gate.p) hipLaunchKernelGGL((gated_norm_backward_kernel<T, NT, NP, true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_norm_backward_kernel<T, NT, NP, false, true>), grid, block, 0, st, a);
  } else {
    if (a.gate.p) hipLaunchKernelGGL((gated_norm_backward_kernel<T, NT, NP, true, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_norm_backward_kernel<T, NT, NP, false, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

// Threads that share a group of so many pieces: as few lanes as hold it with one piece each, up to a wave.  Past
// that the forward pass takes 2 pieces a lane of a wave (with residual and next norm, 32768 x 700 bfloat16
// 55 us; one piece of 128 threads 72), then a workgroup with up to 4 pieces a thread (16384 x 2048: 61; a wave with 4
// pieces a lane 67); the backward pass, with seven rows' pieces at hand, one piece a thread (95; by waves 230).
int threads_of(int pieces, bool back) {
  if (pieces <= 64) {
    int nt = 8;
    while (nt < pieces) nt *= 2;
    return nt;
  }
  if (back) return pieces <= 128 ? 128 : pieces <= 256 ? 256 : pieces <= 512 ? 512 : 1024;
  return pieces <= 128 ? 64 : pieces <= 1024 ? 256 : 1024;
}

template <typename T>
hipError_t pick(const GatedNormArgs& a, bool back, hipStream_t st) {
  const int pieces = (a.D + Piece<T>::N - 1) / Piece<T>::N, nt = threads_of(pieces, back);
  if (back) {
    switch (nt) {
      case 8: return backward<T, 8, 1>(a, st);
      case 16: return backward<T, 16, 1>(a, st);
      case 32: return backward<T, 32, 1>(a, st);
      case 64: return backward<T, 64, 1>(a, st);
      case 128: return backward<T, 128, 1>(a, st);
      case 256: return backward<T, 256, 1>(a, st);
      case 512: return backward<T, 512, 1>(a, st);
      default:
        if (pieces <= 1024) return backward<T, 1024, 1>(a, st);
        // (16384 bfloat16 values are 2048 pieces)
        if constexpr (sizeof(T) == 4)
          if (pieces > 2048) return backward<T, 1024, 4>(a, st);
        return backward<T, 1024, 2>(a, st);
    }
  }
  switch (nt) {
    case 8: return forward<T, 8, 1>(a, st);
    case 16: return forward<T, 16, 1>(a, st);
    case 32: return forward<T, 32, 1>(a, st);
    case 64:
      if (pieces <= 64) return forward<T, 64, 1>(a, st);
      return forward<T, 64, 2>(a, st);
    case 256:
      if (pieces <= 256) return forward<T, 256, 1>(a, st);
      if (pieces <= 512) return forward<T, 256, 2>(a, st);
      return forward<T, 256, 4>(a, st);
    default:
      if constexpr (sizeof(T) == 4)
        if (pieces > 2048) return forward<T, 1024, 4>(a, st);
      return forward<T, 1024, 2>(a, st);
  }
}

}  // namespace

void plan_gated_norm(GatedNormArgs& a, int dtype, bool backward) {
  const int N = dtype == DLA_BF16 ? 8 : 4, pieces = (a.D + N - 1) / N, nt = threads_of(pieces, backward);
  const int per = nt > 256 ? 1 : 256 / nt, side = a.G < per ? a.G : per, along = per / side;
  a.gcols = (a.G + per - 1) / per;
  a.groups = (a.rows + along - 1) / along;
  // The forward pass: a workgroup for every row, up to what a launch takes.  The backward pass, which leaves a
  // part of dw a workgroup: as many as are there at once, and not one more.
  // (8192 forward, which go on to other rows: 65536 x 16 heads of 128 bfloat16 174 us, one row each 215, 2048
  // workgroups 200)
  const bool both = a.gate.p && a.w2 && a.y.p;
  const int waves = dtype == DLA_BF16 ? waves_of<bf16_t>(nt, both) : waves_of<float>(nt, both);
  const int64_t slots = !backward ? 8192 : waves * 256 / (nt > 256 ? nt / 256 : 1);
  const int64_t most = slots / a.gcols > 0 ? slots / a.gcols : 1;
  if (a.groups > most) a.groups = most;
}

int64_t gated_norm_dw_parts(const GatedNormArgs& a) { return a.per_group ? a.groups : a.groups * a.gcols; }

hipError_t launch_gated_norm(const GatedNormArgs& a, int dtype, bool backward, hipStream_t st) {
  return dtype == DLA_BF16 ? pick<bf16_t>(a, backward, st) : pick<float>(a, backward, st);
}

hipError_t launch_gated_norm_dw(const GatedNormArgs& a, float* dw, float* dw2, hipStream_t st) {
  const PartSum p0{a.dw_part, a.rows ? gated_norm_dw_parts(a) : 0, a.per_group ? (int64_t)a.G * a.D : a.D, dw};
  // (the kernel leaves parts of the next norm's weight where it goes through that norm)
  const PartSum p1{a.dw2_part, a.rows && a.y.p ? a.groups * a.gcols : 0, a.D, dw2};
  const unsigned blocks0 = dw ? (unsigned)((p0.width + 31) / 32) : 0, blocks1 = dw2 ? (unsigned)((p1.width + 31) / 32) : 0;
  hipLaunchKernelGGL(part_sum_kernel, dim3(blocks0 + blocks1), dim3(1024), 0, st, p0, p1, blocks0);
  return hipGetLastError();
}

}  // namespace dla
