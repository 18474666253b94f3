// Log probabilities of rows of logits: logprob of a token, entropy, the largest with their indices;
// and the gradient with respect to the logits.
//
// NT threads share a row.  With m the largest logit and s = sum over the others of exp(l - m):
//   lse = m + log(1 + s),  entropy = log(1 + s) + sum exp(l - m) (m - l) / (1 + s)
// so that a probability near one costs no digits.  A row that NT threads hold in registers is read
// once; a longer one is read again from the caches.  Bytes bound the loss, and the gradient,
// which reads and writes a row.
//
// The largest: every thread's largest gives a bound, the top-th largest of those, that at least
// `top` logits reach and few others do; those that reach it are collected in LDS and each counts
// the larger ones.  Logits are compared as 64-bit keys, value first, lower index next, so that no
// two are equal and the order in which they are collected does not matter.
#include "logprobs.h"
#include "piece.h"

namespace dla {
namespace {

constexpr float kInf = __builtin_huge_valf();

// Larger for larger logits, of equal ones for the lower index; above zero.
__device__ __forceinline__ uint64_t key_of(float l, int i) {
  const uint32_t u = __float_as_uint(l + 0.f);   // -0 is 0
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}

template <int NT, typename V, typename F>
__device__ __forceinline__ V over_row(V x, V* lds, F both) {
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

constexpr int kCandidates = 1024;

// The pieces of a row that a thread has: all in registers (NP > 0), or read where they are needed.
template <typename T, int NT, int NP>
struct Row {
  static constexpr int N = Piece<T>::N;
  typename Piece<T>::Raw raw[NP ? NP : 1];
  const T* l;
  int V;
  __device__ __forceinline__ Row(const T* l_, int V_) : l(l_), V(V_) {
    if constexpr (NP > 0) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (i * NT + (int)threadIdx.x) * N;
        raw[i] = Piece<T>::raw(l + c, V > c ? V - c : 0);
      }
    }
  }
  // f(first index, values, elements there are)
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    float x[N];
    if constexpr (NP > 0) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (i * NT + (int)threadIdx.x) * N;
        if (c < V) {
#pragma unroll
          for (int j = 0; j < N; ++j) x[j] = Piece<T>::value(raw[i], j);
          f(c, x, V - c);
        }
      }
    } else {
      for (int64_t c = (int64_t)threadIdx.x * N; c < V; c += NT * N) {
        Piece<T>::load(l + c, V - (int)c, x);
        f((int)c, x, V - (int)c);
      }
    }
  }
};

template <typename T, int NT, int NP, bool TOP>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobArgs a) {
  constexpr int N = Piece<T>::N, NG = NT > 256 ? 256 : NT;
  __shared__ float fl[NT / 64];
  __shared__ uint64_t kl[NT / 64];
  __shared__ uint64_t group[TOP ? NG : 1], cand[TOP ? kCandidates : 1];
  __shared__ uint64_t bound;
  __shared__ int count;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* l = static_cast<const T*>(a.l) + row * a.st;
    const Row<T, NT, NP> r(l, a.V);
    float m = -kInf;
    uint64_t best = 0;
    r.each([&](int c, const float(&x)[N], int n) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j < n) {
          m = fmaxf(m, x[j]);
          if constexpr (TOP) {
            const uint64_t k = key_of(x[j], c + j);
            best = k > best ? k : best;
          }
        }
      }
    });
    m = over_row<NT>(m, fl, [](float p, float q) { return fmaxf(p, q); });
    // the others' sum, those equal to the largest counted
    float s = 0.f, e = 0.f, same = 0.f;
    const float base = m == -kInf ? 0.f : m;     // (a row of -inf alone: all differences -inf)
    r.each([&](int c, const float(&x)[N], int n) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j < n) {
          const float d = x[j] - base, p = __expf(d);
          if (x[j] == m) {
            same += 1.f;
          } else {
            s += p;
            if (p > 0.f || d != d) e -= p * d;     // (p = 0 where d is -inf)
          }
        }
      }
    });
    auto plus = [](float p, float q) { return p + q; };
    s = over_row<NT>(s, fl, plus);
    same = over_row<NT>(same, fl, plus);
    if (a.ent) e = over_row<NT>(e, fl, plus);
    const bool none = m == -kInf && s == 0.f;        // (s is NaN where a logit is)
    s += same - 1.f;
    float ls = log1pf(s);
    if (m == kInf) ls = s = __builtin_nanf("");
    if (threadIdx.x == 0) {
      if (a.lse) a.lse[row] = none ? -kInf : m + ls;
      if (a.ent) a.ent[row] = none ? 0.f : ls + e / (1.f + s);
      if (a.lp) {
        const int64_t t = a.tokens[row];
        float lp = 0.f;
        if (t >= a.V) lp = __builtin_nanf("");
        else if (t >= 0) lp = none ? -kInf : (to_f32(l[t]) - m) - ls;
        a.lp[row] = lp;
      }
    }
    if constexpr (TOP) {
      // the bound: the top-th largest of the groups' largest (zero, which all reach, where there are
      // fewer groups of any)
#pragma unroll
      for (int o = 1; o < NT / NG; o <<= 1) {
        const uint64_t k = __shfl_xor(best, o);
        best = k > best ? k : best;
      }
      __syncthreads();
      if (threadIdx.x % (NT / NG) == 0) group[threadIdx.x / (NT / NG)] = best;
      if (threadIdx.x == 0) {
        count = 0;
        bound = 0;
      }
      __syncthreads();
      if (threadIdx.x < NG) {
        const uint64_t mine = group[threadIdx.x];
        int larger = 0;
        for (int i = 0; i < NG; ++i) larger += group[i] > mine;
        if (mine && larger == a.top - 1) bound = mine;
      }
      __syncthreads();
      const uint64_t b = bound;
      r.each([&](int c, const float(&x)[N], int n) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < n) {
            const uint64_t k = key_of(x[j], c + j);
            if (k >= b) {
              const int at = atomicAdd(&count, 1);
              if (at < kCandidates) cand[at] = k;
            }
          }
      });
      __syncthreads();
      const int found = count;
      auto put = [&](int rank, uint64_t k) {
        a.ids[row * a.top + rank] = index_of(k);
        a.tops[row * a.top + rank] = none ? -kInf : (logit_of(k) - m) - ls;
      };
      if (found <= kCandidates) {
        for (int i = threadIdx.x; i < found; i += NT) {
          const uint64_t mine = cand[i];
          int larger = 0;
          for (int j = 0; j < found; ++j) larger += cand[j] > mine;
          if (larger < a.top) put(larger, mine);
        }
      } else {
        // more reach the bound than there is room for: one after the other
        uint64_t last = ~0ull;
        for (int rank = 0; rank < a.top; ++rank) {
          uint64_t k = 0;
          r.each([&](int c, const float(&x)[N], int n) {
#pragma unroll
            for (int j = 0; j < N; ++j)
              if (j < n) {
                const uint64_t q = key_of(x[j], c + j);
                if (q < last && q > k) k = q;
              }
          });
          last = over_row<NT>(k, kl, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
          if (threadIdx.x == 0) put(rank, last);
        }
      }
      __syncthreads();
    }
  }
}

// dl_i = p_i (dlse - dlp - dent (log p_i + entropy)) + [i = token] dlp
template <typename T>
__global__ __launch_bounds__(256) void logprob_backward_kernel(LogprobArgs a, int cols) {
  constexpr int N = Piece<T>::N, NP = 4;
  const int64_t blocks = a.rows * cols;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t row = block / cols;
    const int64_t c0 = (block % cols) * (256 * NP * N);
    const T* l = static_cast<const T*>(a.l) + row * a.st;
    T* dl = static_cast<T*>(a.dl) + row * a.dst;
    typename Piece<T>::Raw raw[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t c = c0 + (i * 256 + (int)threadIdx.x) * N;
      raw[i] = Piece<T>::raw(l + c, a.V > c ? (int)(a.V - c) : 0);
    }
    const int64_t t = a.tokens ? a.tokens[row] : -1;
    const float lse = a.lse[row], dent = a.dent ? a.dent[row] : 0.f, ent = a.dent ? a.ent[row] : 0.f;
    float dlp = a.dlp && t >= 0 ? a.dlp[row] : 0.f;
    const float dlse = a.dlse ? a.dlse[row] : 0.f;
    const bool none = lse == -kInf;    // a row of -inf alone
    const float at = a.dlp && t >= 0 && t < a.V && !none ? -dlp * expm1f(a.lp[row]) : 0.f;   // dlp (1 - p), to its last digits
    if (a.dlp && t >= a.V) dlp = __builtin_nanf("");
    const float k = dlse - dlp;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t c = c0 + (i * 256 + (int)threadIdx.x) * N;
      float x[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float lp = Piece<T>::value(raw[i], j) - lse, p = __expf(lp);
        float f = c + j == t ? dlse : k;
        if (a.dent) f -= dent * (lp + ent);
        x[j] = (p == 0.f || none ? (k != k ? k : 0.f) : p * f) + (c + j == t ? at : 0.f);
      }
      if (c < a.V) Piece<T>::store(dl + c, (int)(a.V - c < N ? a.V - c : N), x);
    }
  }
}

template <typename T, int NT, int NP>
hipError_t go(const LogprobArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20)), block(NT);
  if (a.top) hipLaunchKernelGGL((logprob_kernel<T, NT, NP, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((logprob_kernel<T, NT, NP, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t pick(const LogprobArgs& a, hipStream_t st) {
  const int pieces = (int)(((int64_t)a.V + Piece<T>::N - 1) / Piece<T>::N);
  if (pieces <= 128) return go<T, 64, 2>(a, st);
  if (pieces <= 1024) return go<T, 256, 4>(a, st);
  if (pieces <= 4096) return go<T, 1024, 4>(a, st);
  if (pieces <= 8192) return go<T, 1024, 8>(a, st);
  return go<T, 1024, 0>(a, st);
}

template <typename T>
hipError_t back(const LogprobArgs& a, hipStream_t st) {
  const int per = 256 * 4 * Piece<T>::N, cols = (int)(((int64_t)a.V + per - 1) / per);
  const int64_t blocks = a.rows * cols;
  hipLaunchKernelGGL((logprob_backward_kernel<T>), dim3((unsigned)(blocks < (1 << 23) ? blocks : 1 << 23)), dim3(256), 0,
                     st, a, cols);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t st) {
  return dtype == DLA_BF16 ? pick<bf16_t>(a, st) : pick<float>(a, st);
}

hipError_t launch_logprobs_backward(const LogprobArgs& a, int dtype, hipStream_t st) {
  return dtype == DLA_BF16 ? back<bf16_t>(a, st) : back<float>(a, st);
}

}  // namespace dla
