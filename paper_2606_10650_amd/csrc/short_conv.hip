// The short causal convolution: z_t = bias + sum_j w_j x_{t - (W - 1) + j} per channel, y = silu(z);
// and its backward pass.
//
// A thread holds a piece of channels (16 bytes of a row) with their taps in registers and walks
// along a run of tokens with the last W - 1 inputs in registers too, so that an input is read
// once but for the W - 1 in front of a run.  A document's start clears those registers.  The
// backward pass forms z again and carries the W - 1 gradients that are not yet whole; behind its
// run it reads W - 1 tokens more.
//
// Bytes bound both passes: 4 x 16384 tokens of 6144 bfloat16 channels, forward 1.6 GB and backward 2.4 GB, take
// 830 us together, 4.9 TB/s of the 5.1 that a copy reaches.  So that the next group of tokens is on its way while
// one is worked on, all that it needs comes with it, the starts of documents too (read token by token, each
// waited for behind the loads of the next group: 1024 us), and backward a group inside its run and its
// document goes without the checks of the others (872).  A run's taps come by whole pieces (one by one 850;
// one token of 64 sequences 5.4 us, one by one 8.4).  The backward pass has registers for two waves a SIMD;
// channels by fours, for twice the waves, took a fifth longer.
#include <type_traits>

#include "piece.h"
#include "short_conv.h"

namespace dla {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

__device__ __forceinline__ int length_of(const ConvArgs& a, int b) {
  if (!a.lengths) return a.T;
  const int n = a.lengths[b];
  return n < 0 ? 0 : (n > a.T ? a.T : n);
}

// Taps and bias of a piece of channels.
template <typename T, int W>
struct Taps {
  static constexpr int N = Piece<T>::N;
  float w[W][N], bias[N];
  __device__ __forceinline__ void load(const ConvArgs& a, int c, int n) {
    if (a.w_f32) load_as<float>(a, c, n);
    else load_as<T>(a, c, n);
#pragma unroll
    for (int i = 0; i < N; ++i) bias[i] = 0.f;
    if (a.bias) load_floats<T>(a.bias, a.w_f32, c, n, bias);
  }
  // the channels' taps lie one after the other, and come by pieces of 16 bytes
  template <typename S>
  __device__ __forceinline__ void load_as(const ConvArgs& a, int c, int n) {
    using P = Piece<S>;
    const S* from = static_cast<const S*>(a.w) + (int64_t)c * W;
    const int all = min(n, N) * W;
    typename P::Raw raw[N * W / P::N];
#pragma unroll
    for (int q = 0; q < N * W / P::N; ++q) raw[q] = P::raw(from + q * P::N, all - q * P::N);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = P::value(raw[(i * W + j) / P::N], (i * W + j) % P::N);
  }
};

// The W - 1 inputs before a token, the latest last.
template <typename T, int W>
struct Window {
  static constexpr int N = Piece<T>::N;
  float x[W - 1][N];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) x[j][i] = 0.f;
  }
  __device__ __forceinline__ void push(const float (&v)[N]) {
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) x[j][i] = x[j + 1][i];
#pragma unroll
    for (int i = 0; i < N; ++i) x[W - 2][i] = v[i];
  }
  // What token t of sequence b sees before its own start is looked at: asked for, all of it before any is waited
  // for, and taken.
  struct Before {
    typename Piece<T>::Raw raw[W - 1];
    uint8_t start[W - 1];
    __device__ __forceinline__ void fetch(const ConvArgs& a, int b, int t, int c, int n) {
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        const int p = t - (W - 1) + j;
        const T* from = p >= 0 ? static_cast<const T*>(a.x.p) + b * a.x.sb + p * a.x.st + c
                        : a.state ? static_cast<const T*>(a.state) + ((int64_t)b * (W - 1) + W - 1 + p) * a.C + c
                                  : nullptr;
        raw[j] = {};
        if (from) raw[j] = Piece<T>::raw(from, n);
        start[j] = 0;
        if (p >= 0 && a.starts) start[j] = a.starts[(int64_t)b * a.T + p];
      }
    }
  };
  // Returns how many inputs before t its document has (W - 1: all there are room for).
  __device__ __forceinline__ int take(const Before& o) {
    clear();
    int age = W - 1;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      if (o.start[j]) {
        clear();
        age = W - 1 - j;
      }
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = Piece<T>::value(o.raw[j], i);
      push(v);
    }
    return age;
  }
};

template <typename T, int W>
__device__ __forceinline__ void convolve(const Taps<T, W>& k, const Window<T, W>& win,
                                         const float (&x)[Piece<T>::N], float (&z)[Piece<T>::N]) {
#pragma unroll
  for (int i = 0; i < Piece<T>::N; ++i) {
    z[i] = k.bias[i];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) z[i] += k.w[j][i] * win.x[j][i];
    z[i] += k.w[W - 1][i] * x[i];
  }
}

// Where a thread works: a piece of channels of a run of tokens of a sequence.
struct Place {
  int b, c, t0, t1;
  bool any;
};

// A workgroup has `lanes` pieces side by side and 256 / lanes runs; one of the backward pass goes
// on to the runs `pass` times all workgroups' on.
__device__ __forceinline__ Place place_of(const ConvArgs& a, int N, int64_t pass) {
  const int cols = (a.pieces + a.lanes - 1) / a.lanes, runs = 256 / a.lanes;
  const int64_t run = (pass * a.groups + blockIdx.x / cols) * runs + threadIdx.x / a.lanes;
  const int piece = (int)(blockIdx.x % cols) * a.lanes + threadIdx.x % a.lanes;
  Place p;
  p.any = run < (int64_t)a.B * a.chunks && piece < a.pieces;
  p.b = (int)(run / a.chunks);
  p.t0 = (int)(run % a.chunks) * a.per;
  p.t1 = min(p.t0 + a.per, a.T);
  p.c = piece * N;
  return p;
}

template <typename T, int W>
__global__ __launch_bounds__(256) void conv_kernel(ConvArgs a) {
  constexpr int N = Piece<T>::N, G = 4;
  using Raw = typename Piece<T>::Raw;
  const Place p = place_of(a, N, 0);
  if (!p.any) return;
  const int n = a.C - p.c, len = length_of(a, p.b), end = min(p.t1, len);
  const T* x = static_cast<const T*>(a.x.p) + p.b * a.x.sb + p.c;
  T* y = static_cast<T*>(a.y.p) + p.b * a.y.sb + p.c;
  const uint8_t* starts = a.starts ? a.starts + (int64_t)p.b * a.T : nullptr;
  // groups of tokens, the next group's on its way; behind the last token the last one again
  Raw next[G];
  uint8_t start[G] = {};
  auto fetch = [&](int t) {
    if (starts)
#pragma unroll
      for (int g = 0; g < G; ++g) start[g] = starts[min(t + g, end - 1)];
#pragma unroll
    for (int g = 0; g < G; ++g) next[g] = Piece<T>::raw(x + min(t + g, end - 1) * a.x.st, n);
  };
  // all that the first token needs is asked for before any is waited for
  Window<T, W> win;
  typename Window<T, W>::Before before = {};
  // (a run behind the sequence's end has nothing before it, and must not read the state)
  if (p.t0 < len || p.t0 == 0) before.fetch(a, p.b, p.t0, p.c, n);
  if (p.t0 < end) fetch(p.t0);
  Taps<T, W> k;
  k.load(a, p.c, n);
  win.take(before);
  for (int t = p.t0; t < end; t += G) {
    Raw raw[G];
    uint8_t first[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      raw[g] = next[g];
      first[g] = start[g];
    }
    if (t + G < end) fetch(t + G);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (t + g < end) {
        float v[N], z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = Piece<T>::value(raw[g], i);
        if (first[g]) win.clear();
        convolve<T, W>(k, win, v, z);
        win.push(v);
        if (a.silu) {
#pragma unroll
          for (int i = 0; i < N; ++i) z[i] *= sigmoid(z[i]);
        }
        Piece<T>::store(y + (t + g) * a.y.st, n, z);
      }
    }
  }
  if (end < p.t1) {
    const float zero[N] = {};
    for (int t = max(p.t0, end); t < p.t1; ++t) Piece<T>::store(y + t * a.y.st, n, zero);
  }
  // the first run's thread alone has read the given state, and writes the last one over it
  if (a.state_out && p.t0 == 0) {
    if (len > end) {
      before.fetch(a, p.b, len, p.c, n);
      win.take(before);
    }
    T* s = static_cast<T*>(a.state_out) + (int64_t)p.b * (W - 1) * a.C + p.c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) Piece<T>::store(s + (int64_t)j * a.C, n, win.x[j]);
  }
}

template <typename T, int W>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvArgs a) {
  constexpr int N = Piece<T>::N, G = sizeof(T) == 2 ? 2 : 4;
  using Raw = typename Piece<T>::Raw;
  __shared__ float sums[256 * N];
  const int n = a.C - ((int)(blockIdx.x % ((a.pieces + a.lanes - 1) / a.lanes)) * a.lanes + (int)threadIdx.x % a.lanes) * N;
  Taps<T, W> k;
  if (n > 0) k.load(a, a.C - n, n);
  float dw[W + 1][N];
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) dw[j][i] = 0.f;
  for (int64_t pass = 0; pass < a.passes; ++pass) {
    const Place p = place_of(a, N, pass);
    if (!p.any) break;
    const int len = length_of(a, p.b);
    const T* x = static_cast<const T*>(a.x.p) + p.b * a.x.sb + p.c;
    const T* dy = static_cast<const T*>(a.y.p) + p.b * a.y.sb + p.c;
    T* dx = static_cast<T*>(a.dx.p) + p.b * a.dx.sb + p.c;
    const uint8_t* starts = a.starts ? a.starts + (int64_t)p.b * a.T : nullptr;
    Window<T, W> win;
    typename Window<T, W>::Before before;
    before.fetch(a, p.b, min(p.t0, len), p.c, n);
    int age;
    float pend[W - 1][N];   // gradients of the W - 1 inputs before, the latest last
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) pend[j][i] = 0.f;
    T* ds = a.dstate ? static_cast<T*>(a.dstate) + (int64_t)p.b * (W - 1) * a.C + p.c : nullptr;
    // the gradient of input q of the sequence is whole
    auto put = [&](int q, const float(&v)[N]) {
      if (q >= p.t0 && q < p.t1) Piece<T>::store(dx + q * a.dx.st, n, v);
      else if (q < 0 && p.t0 == 0 && ds) Piece<T>::store(ds + (int64_t)(W - 1 + q) * a.C, n, v);
    };
    const int last = min(min(p.t1, a.T - (W - 1)) + W - 1, len);   // t1 + W - 1 without leaving int32
    // WHOLE: the run's own token, all inputs that it sees of its document and of the run
    auto token = [&](int t, const Raw& rawx, const Raw& rawd, bool first, auto kind) {
      constexpr bool WHOLE = decltype(kind)::value;
      float v[N], z[N], d[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = Piece<T>::value(rawx, i);
        d[i] = Piece<T>::value(rawd, i);
      }
      if (!WHOLE && first) {
        win.clear();
        age = 0;
      }
      if (a.silu) {
        convolve<T, W>(k, win, v, z);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float s = sigmoid(z[i]);
          d[i] *= s * (1.f + z[i] * (1.f - s));
        }
      }
      if (WHOLE || t < p.t1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          dw[W][i] += d[i];
          dw[W - 1][i] += d[i] * v[i];
#pragma unroll
          for (int j = 0; j < W - 1; ++j) dw[j][i] += d[i] * win.x[j][i];
        }
      }
      win.push(v);
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (WHOLE || W - 1 - j <= age) {
#pragma unroll
          for (int i = 0; i < N; ++i) pend[j][i] += k.w[j][i] * d[i];
        }
      if constexpr (WHOLE) {
        Piece<T>::store(dx + (int64_t)(t - (W - 1)) * a.dx.st, N, pend[0]);
      } else {
        age = min(age + 1, W - 1);
        put(t - (W - 1), pend[0]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) pend[j][i] = pend[j + 1][i];
        pend[W - 2][i] = k.w[W - 1][i] * d[i];
      }
    };
    // groups of tokens, the next group's on its way; behind the last token the last one again
    Raw rx[G], rd[G];
    uint8_t rs[G] = {};
    auto fetch = [&](int t) {
      if (starts)
#pragma unroll
        for (int g = 0; g < G; ++g) rs[g] = starts[min(t + g, last - 1)];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int64_t q = min(t + g, last - 1);
        rx[g] = Piece<T>::raw(x + q * a.x.st, n);
        rd[g] = Piece<T>::raw(dy + q * a.y.st, n);
      }
    };
    if (p.t0 < last) fetch(p.t0);
    // (inputs of before the run have their gradients from the run before, but for the state's)
    age = win.take(before);
    for (int t = p.t0; t < last; t += G) {
      Raw cx[G], cd[G];
      uint8_t first[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        cx[g] = rx[g];
        cd[g] = rd[g];
        first[g] = rs[g];
      }
      if (t + G < last) fetch(t + G);
      bool whole = n >= N && age == W - 1 && t - (W - 1) >= p.t0 && t + G <= last && t + G <= p.t1;
#pragma unroll
      for (int g = 0; g < G; ++g) whole = whole && !first[g];
      if (whole) {
#pragma unroll
        for (int g = 0; g < G; ++g) token(t + g, cx[g], cd[g], false, std::true_type());
      } else {
#pragma unroll
        for (int g = 0; g < G; ++g)
          if (t + g < last) token(t + g, cx[g], cd[g], first[g], std::false_type());
      }
    }
    const int t = max(p.t0, last);   // the token behind those that were looked at
    if (p.t0 <= len) {
      // the sequence's end: what the last state's gradient asks of the inputs that it shows
      if (t == len && a.dstate_out) {
        const T* g = static_cast<const T*>(a.dstate_out) + (int64_t)p.b * (W - 1) * a.C + p.c;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
          if (W - 1 - j <= age) {
            float v[N];
            Piece<T>::load(g + (int64_t)j * a.C, n, v);
#pragma unroll
            for (int i = 0; i < N; ++i) pend[j][i] += v[i];
          }
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) put(t - (W - 1) + j, pend[j]);
    }
    const float zero[N] = {};
    for (int q = max(p.t0, len); q < p.t1; ++q) Piece<T>::store(dx + q * a.dx.st, n, zero);
  }
  if (!a.part) return;
  // the workgroup's runs one after the other into one sum
  const int runs = 256 / a.lanes, lane = threadIdx.x % a.lanes;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    if (runs > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) sums[i * 256 + threadIdx.x] = dw[j][i];
      __syncthreads();
      if (threadIdx.x < (unsigned)a.lanes) {
        for (int r = 1; r < runs; ++r)
#pragma unroll
          for (int i = 0; i < N; ++i) dw[j][i] += sums[i * 256 + r * a.lanes + lane];
      }
    }
  }
  const int cols = (a.pieces + a.lanes - 1) / a.lanes;
  const int piece = (int)(blockIdx.x % cols) * a.lanes + lane;
  if (threadIdx.x < (unsigned)a.lanes && piece < a.pieces) {
    float* part = a.part + ((int64_t)(blockIdx.x / cols) * a.C + piece * N) * (W + 1);
    const int all = min(n, N) * (W + 1);
#pragma unroll
    for (int q = 0; q < N * (W + 1); q += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = dw[(q + e) % (W + 1)][(q + e) / (W + 1)];
      Piece<float>::store(part + q, all - q, v);
    }
  }
}

// dw and dbias from the workgroups' parts: 32 columns a workgroup, 32 threads to a column, in a fixed order, in
// float64
__global__ __launch_bounds__(1024) void conv_sum_kernel(const float* part, int64_t parts, int C, int W, float* dw, float* db) {
  __shared__ double sums[32][33];
  const int col = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t width = (int64_t)C * (W + 1), at = (int64_t)blockIdx.x * 32 + col;
  double s = 0.;
  if (at < width) {
    int64_t i = r;
    for (; i + 96 < parts; i += 128) {
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = part[(i + 32 * j) * width + at];
      s += ((double)x[0] + x[1]) + ((double)x[2] + x[3]);
    }
    for (; i < parts; i += 32) s += part[i * width + at];
  }
  sums[r][col] = s;
  __syncthreads();
  if (r == 0 && at < width) {
    for (int i = 1; i < 32; ++i) s += sums[i][col];
    const int c = (int)(at / (W + 1)), j = (int)(at % (W + 1));
    if (j < W) dw[(int64_t)c * W + j] = (float)s;
    else if (db) db[c] = (float)s;
  }
}

template <typename T, int W>
hipError_t go(const ConvArgs& a, bool backward, float* dw, float* db, hipStream_t st) {
  const int cols = (a.pieces + a.lanes - 1) / a.lanes;
  const dim3 grid((unsigned)(cols * a.groups)), block(256);
  if (!backward) {
    if (grid.x) hipLaunchKernelGGL((conv_kernel<T, W>), grid, block, 0, st, a);
  } else {
    if (grid.x) hipLaunchKernelGGL((conv_backward_kernel<T, W>), grid, block, 0, st, a);
    if (dw && a.C) {
      const int64_t width = (int64_t)a.C * (W + 1);
      hipLaunchKernelGGL(conv_sum_kernel, dim3((unsigned)((width + 31) / 32)), dim3(1024), 0, st, a.part,
                         a.groups, a.C, W, dw, db);
    }
  }
  return hipGetLastError();
}

hipError_t pick(const ConvArgs& a, int dtype, bool backward, float* dw, float* db, hipStream_t st) {
  if (dtype == DLA_BF16) {
    if (a.W == 2) return go<bf16_t, 2>(a, backward, dw, db, st);
    if (a.W == 3) return go<bf16_t, 3>(a, backward, dw, db, st);
    return go<bf16_t, 4>(a, backward, dw, db, st);
  }
  if (a.W == 2) return go<float, 2>(a, backward, dw, db, st);
  if (a.W == 3) return go<float, 3>(a, backward, dw, db, st);
  return go<float, 4>(a, backward, dw, db, st);
}

}  // namespace

// Runs.  4 x 16384 tokens of 6144 bfloat16 channels, backward: 504 workgroups, all there at once; 516, four more
// than there is room for, took 1.6 times as long, twice as many, each half as long, 1.06 times.
void plan_conv(ConvArgs& a, int dtype, bool backward) {
  const int N = dtype == DLA_BF16 ? 8 : 4;
  a.pieces = (int)(((int64_t)a.C + N - 1) / N);
  a.lanes = 64;
  while (a.lanes > 1 && a.lanes / 2 >= a.pieces) a.lanes /= 2;
  const int64_t cols = (a.pieces + a.lanes - 1) / a.lanes, each = 256 / a.lanes;
  if (a.B == 0 || a.pieces == 0) {
    a.chunks = a.passes = a.per = 1;
    a.groups = 0;
    return;
  }
  // Workgroups at once: of the backward pass as many as its registers let be there, and not one more.
  int64_t groups = (backward ? 512 : 1024) / cols;
  if (groups < 1) groups = 1;
  // tokens a run, so that all runs are there at once; 8 at least, and forward, where no sums are kept, 64 at
  // most
  const int64_t share = groups * each / a.B;
  int64_t per = share > 0 ? ((int64_t)a.T + share - 1) / share : a.T;
  if (per < 8) per = 8;
  if (!backward && per > 64) per = 64;
  if (per > a.T) per = a.T > 0 ? a.T : 1;
  a.per = (int)per;
  a.chunks = a.T > 0 ? (int)(((int64_t)a.T + per - 1) / per) : 1;
  const int64_t all = ((int64_t)a.B * a.chunks + each - 1) / each;
  a.passes = backward ? (int)((all + groups - 1) / groups) : 1;
  a.groups = (all + a.passes - 1) / a.passes;
}

hipError_t launch_conv(const ConvArgs& a, int dtype, hipStream_t st) {
  return pick(a, dtype, false, nullptr, nullptr, st);
}

hipError_t launch_conv_backward(const ConvArgs& a, int dtype, float* dw, float* db, hipStream_t st) {
  return pick(a, dtype, true, dw, db, st);
}

}  // namespace dla
