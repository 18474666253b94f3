// Log probabilities of rows of logits: logprob of a token, entropy, the largest with their indices;
// and the gradient with respect to the logits.
//
// A row is read once.  NT threads go through it, each with the largest logit that it has met and the
// sum of the others' exponentials: of a new logit and the largest so far the lower one joins the
// sum.  So the largest one's own term is never in it, and with m the largest, s the sum of the
// others' exp(l - m),
//   lse = m + log(1 + s),  entropy = log(1 + s) + sum exp(l - m) (m - l) / (1 + s)
// a probability near one costs no digits.  Exponentials are taken relative to the largest of the row's
// first logits, and the sums scaled afterwards; where the row's largest is further than 2^24 times as
// likely as that, the row is read again (from the caches) with its own.  Bytes bound the loss, and the gradient,
// which reads and writes a row; the exponentials and the sums take nearly as long as the bytes.  8192 rows of
// 50304 bfloat16: 155 us, 5.3 TB/s, with entropies 187, 4.4, the gradient 286, 5.8.  (A row held in the
// registers of 1024 threads, its largest found first: 436.)
//
// Few long rows are worked on in parts, which a second kernel joins.
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

constexpr int kCandidates = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// The pieces of a run of n logits that a thread of NT has, in groups of G: first the groups that lie inside
// as a whole, then the rest.  Of the rest the last piece starts N elements before the end, with those
// that the piece before it has, and all of pieces behind the end, as -inf: every load is a whole
// piece, without a branch around it.
template <typename T, int NT>
struct Run {
  static constexpr int N = Piece<T>::N, G = 2, GROUP = G * NT * N;
  using Raw = typename Piece<T>::Raw;
  const T* l;
  int n, whole;    // whole groups
  __device__ __forceinline__ Run(const T* l_, int n_) : l(l_), n(n_), whole(n_ / GROUP) {}
  __device__ __forceinline__ int first(int group, int g) const { return group * GROUP + (g * NT + (int)threadIdx.x) * N; }
  __device__ __forceinline__ int start(int64_t c) const { return (int)(c + N <= n ? c : n > N ? n - N : 0); }
  __device__ __forceinline__ void load(Raw (&x)[G], int group) const {
    if (group < whole) {
      const T* p = l + first(group, 0);
#pragma unroll
      for (int g = 0; g < G; ++g) x[g] = *reinterpret_cast<const Raw*>(p + g * NT * N);
      return;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int64_t c = group * (int64_t)GROUP + (g * NT + (int)threadIdx.x) * N, skip = c - start(c);
      if (n >= N) x[g] = *reinterpret_cast<const Raw*>(l + start(c));
      else x[g] = Piece<T>::raw(l, n);    // (the whole run)
      if (c + N <= n) continue;
      // -inf in the elements that are not the piece's own
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < skip || j >= n) {
          if constexpr (sizeof(T) == 2) {
            x[g].w[j >> 1] = (x[g].w[j >> 1] & (0xFFFFu << (16 * (1 - (j & 1))))) | 0xFF80u << (16 * (j & 1));
          } else {
            x[g].w[j] = 0xFF800000u;
          }
        }
    }
  }
  __device__ __forceinline__ int groups() const { return whole + (n > whole * (int64_t)GROUP); }
  // f(piece) for all, x holding the first group's; the next group is on its way
  template <typename F>
  __device__ __forceinline__ void each(Raw (&x)[G], F f) const {
    for (int i = 0; i < whole; ++i) {
      Raw y[G];
      if (i + 1 < groups()) load(y, i + 1);
#pragma unroll
      for (int g = 0; g < G; ++g) f(x[g]);
#pragma unroll
      for (int g = 0; g < G; ++g) x[g] = y[g];
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (whole * (int64_t)GROUP + g * NT * N < n) f(x[g]);
  }
};

// The largest logit, and of the others the sums of p and of -p d, p = 2^d.  d is the logit times log2 e less
// `base`, a whole number: one operation, rounded once.  EXACT: the logit less `base`, another logit, times
// log2 e, for logits whose multiple has no finite value.
template <bool ENT, bool EXACT>
struct Sums {
  float m = -kInf, s = 0.f, e = 0.f;
  __device__ __forceinline__ static float scaled(float x, float base) {
    return EXACT ? (x - base) * kLog2e : __builtin_fmaf(x, kLog2e, -base);
  }
  // A d of -inf (a logit shut out) counts as -2000, whose power is zero too and times it; a NaN is not larger
  // than anything, and joins the sums.
  __device__ __forceinline__ void join(float x, float base) {
    const float low = x > m ? m : x;
    m = fmaxf(m, x);
    const float d = scaled(low, base), p = __builtin_amdgcn_exp2f(d);
    s += p;
    if constexpr (ENT) e -= p * fmaxf(d, -2000.f);
  }
  __device__ __forceinline__ void join(const Sums& o, float base) {
    join(o.m, base);
    s += o.s;
    if constexpr (ENT) e += o.e;
  }
};

// What a run gives: its largest logit, and the others' sums relative to it.
struct Found {
  float m, s, e, mine;    // (and the thread's own largest)
};

// A run by one pass, relative to what is given; false where that is too far from the run's largest.
template <typename T, int NT, bool ENT, bool EXACT>
__device__ __forceinline__ bool pass(const Run<T, NT>& r, typename Piece<T>::Raw (&x)[Run<T, NT>::G], float base,
                                     float (&lds)[4][NT / 64], Found& f) {
  using S = Sums<ENT, EXACT>;
  S t;
  r.each(x, [&](const typename Piece<T>::Raw& piece) {
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j) t.join(Piece<T>::value(piece, j), base);
  });
  f.mine = t.m;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    S u;
    u.m = __shfl_xor(t.m, o);
    u.s = __shfl_xor(t.s, o);
    if constexpr (ENT) u.e = __shfl_xor(t.e, o);
    // (the lower lane's sums first, so that all lanes find the same)
    const bool lower = (threadIdx.x & o) == 0;
    S v = lower ? t : u;
    v.join(lower ? u : t, base);
    t = v;
  }
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      lds[1][threadIdx.x >> 6] = t.m;
      lds[2][threadIdx.x >> 6] = t.s;
      lds[3][threadIdx.x >> 6] = t.e;
    }
    __syncthreads();
    t = S();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      S u;
      u.m = lds[1][i];
      u.s = lds[2][i];
      u.e = lds[3][i];
      t.join(u, base);
    }
  }
  const float d = S::scaled(t.m, base), k = __builtin_amdgcn_exp2f(-d);
  f.m = t.m;
  f.s = t.s;
  f.e = 0.f;
  if (t.m == -kInf) return true;      // (the others too, or NaN)
  f.s = t.s * k;
  f.e = kLn2 * k * (t.e + d * t.s);
  return EXACT || (fabsf(d) <= 24.f && t.s != kInf);
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

// put(rank, key) for the `top` largest of n <= 1024 keys in LDS, no two equal but zeros, which stand for none.
// Up to NT: each key's rank is counted by as many threads as there are; more: four keys a thread.
template <int NT, typename F>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int top, int* ranks, F put) {
  if (n <= NT) {
    const int width = (n + 63) & ~63, shares = NT / width, i = threadIdx.x % width, share = threadIdx.x / width;
    if (shares > 1) {
      for (int j = threadIdx.x; j < n; j += NT) ranks[j] = 0;
      __syncthreads();
    }
    const uint64_t key = i < n && share < shares ? keys[i] : 0;
    int more = 0;
    if (key) {
      const int to = (share + 1) * n / shares;
#pragma unroll 8
      for (int j = share * n / shares; j < to; ++j) more += keys[j] > key;
    }
    if (shares > 1) {
      if (more) atomicAdd(&ranks[i], more);
      __syncthreads();
      if (key && share == 0) more = ranks[i];
    }
    if (key && share == 0 && more < top) put(more, key);
  } else {
    uint64_t key[1024 / NT];
    int more[1024 / NT];
#pragma unroll
    for (int q = 0; q < 1024 / NT; ++q) {
      const int i = q * NT + (int)threadIdx.x;
      key[q] = i < n ? keys[i] : 0;
      more[q] = 0;
    }
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const uint64_t k = keys[j];
#pragma unroll
      for (int q = 0; q < 1024 / NT; ++q) more[q] += k > key[q];
    }
#pragma unroll
    for (int q = 0; q < 1024 / NT; ++q)
      if (key[q] && more[q] < top) put(more[q], key[q]);
  }
}

// A row's results from m, and s and e relative to it.
__device__ __forceinline__ void put_row(const LogprobArgs& a, int64_t row, float m, float ls, float ent, bool none) {
  if (a.lse) a.lse[row] = none ? -kInf : m + ls;
  if (a.ent) a.ent[row] = none ? 0.f : ent;
  if (a.lp) {
    const int64_t t = a.tokens[row];
    float lp = 0.f;
    if (t >= a.V) lp = __builtin_nanf("");
    else if (t >= 0) {
      const float l = a.bf16 ? to_f32(static_cast<const bf16_t*>(a.l)[row * a.st + t]) : static_cast<const float*>(a.l)[row * a.st + t];
      lp = none ? -kInf : (l - m) - ls;
    }
    a.lp[row] = lp;
  }
}

template <typename T, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobArgs a) {
  constexpr int N = Piece<T>::N, G = Run<T, NT>::G;
  using Raw = typename Piece<T>::Raw;
  __shared__ float fl[4][NT / 64];
  __shared__ uint64_t kl[NT / 64];
  __shared__ float group[TOP ? 64 : 1];
  __shared__ uint64_t cand[TOP ? kCandidates : 1];
  __shared__ int ranks[TOP ? NT : 1];
  __shared__ float bound;
  __shared__ int count;
  const int64_t blocks = a.rows * a.parts;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t row = block / a.parts;
    const int part = (int)(block - row * a.parts), first = part * a.per;
    const Run<T, NT> r(static_cast<const T*>(a.l) + row * a.st + first, min(a.per, a.V - first));
    // the largest of the first logits
    Raw x[G];
    r.load(x, 0);
    float base = -kInf;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int j = 0; j < N; ++j) base = fmaxf(base, Piece<T>::value(x[g], j));
    base = over_row<NT>(base, fl[0], [](float p, float q) { return fmaxf(p, q); });
    Found f;
    if (r.groups() == 1) {
      // all of the run is there, and its largest: the others' sums by adding up
      const float zero = base == -kInf ? 0.f : base;
      float s = 0.f, e = 0.f, same = 0.f;
      f.mine = -kInf;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float v = Piece<T>::value(x[g], j), d = (v - zero) * kLog2e;
          const float p = v == base ? 0.f : __builtin_amdgcn_exp2f(d);
          same += v == base ? 1.f : 0.f;
          s += p;
          if constexpr (ENT) e -= p * fmaxf(d, -2000.f);
          if constexpr (TOP) f.mine = fmaxf(f.mine, v);
        }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        s += __shfl_xor(s, o);
        same += __shfl_xor(same, o);
        if constexpr (ENT) e += __shfl_xor(e, o);
      }
      if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) {
          fl[1][threadIdx.x >> 6] = same;
          fl[2][threadIdx.x >> 6] = s;
          fl[3][threadIdx.x >> 6] = e;
        }
        __syncthreads();
        s = e = same = 0.f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) {
          same += fl[1][i];
          s += fl[2][i];
          e += fl[3][i];
        }
      }
      f.m = base;
      f.s = base == -kInf ? s : s + (same - 1.f);
      f.e = kLn2 * e;
    } else {
      const float whole = base == -kInf ? 0.f : rintf(base * kLog2e);
      if (!pass<T, NT, ENT, false>(r, x, whole, fl, f)) {
        r.load(x, 0);
        const float m = f.m;
        pass<T, NT, ENT, true>(r, x, m, fl, f);
      }
    }
    const float m = f.m;
    float s = f.s, e = f.e;
    const bool none = m == -kInf && s == 0.f;        // (s is NaN where a logit is)
    if (m == kInf) s = __builtin_nanf("");
    const float ls = log1pf(s);
    if (threadIdx.x == 0) {
      if (a.parts == 1) {
        put_row(a, row, m, ls, ls + e / (1.f + s), none);
      } else {
        a.part_sums[block * 3] = m;
        a.part_sums[block * 3 + 1] = s;
        a.part_sums[block * 3 + 2] = e;
      }
    }
    if constexpr (TOP) {
      // the bound: the top-th largest of 64 groups' largest
      float best = f.mine;
#pragma unroll
      for (int o = 1; o < NT / 64; o <<= 1) best = fmaxf(best, __shfl_xor(best, o));
      __syncthreads();
      if (threadIdx.x % (NT / 64) == 0) group[threadIdx.x / (NT / 64)] = best;
      if (threadIdx.x == 0) {
        count = 0;
        bound = -kInf;
      }
      __syncthreads();
      if (threadIdx.x < 64) {
        const float mine = group[threadIdx.x];
        int larger = 0, equal = 0;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) {
          larger += group[i] > mine;
          equal += group[i] == mine;
        }
        if (larger < a.top && larger + equal >= a.top) bound = mine;   // (all who find it find the same)
      }
      __syncthreads();
      // (written so that a NaN reaches it)
      const float b = bound;
      for (int i = 0; i < r.groups() && !(f.mine < b); ++i) {
        if (r.groups() > 1) r.load(x, i);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const int64_t own = i * (int64_t)r.GROUP + (g * NT + (int)threadIdx.x) * N, at = r.start(own);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const float v = Piece<T>::value(x[g], j);
            if (!(v < b) && at + j >= own && at + j < r.n) {
              const int place = atomicAdd(&count, 1);
              if (place < kCandidates) cand[place] = key_of(v, first + (int)(at + j));
            }
          }
        }
      }
      __syncthreads();
      const int found = count, want = min(a.top, r.n);
      auto put = [&](int rank, uint64_t key) {
        if (a.parts == 1) {
          a.ids[row * a.top + rank] = index_of(key);
          a.tops[row * a.top + rank] = none ? -kInf : (logit_of(key) - m) - ls;
        } else {
          a.part_keys[block * a.top + rank] = key;
        }
      };
      if (found >= want && found <= kCandidates) {
        rank_keys<NT>(cand, found, a.top, ranks, put);
      } else {
        // more reach the bound than there is room for (or, of a row with NaN, fewer): one after the other
        uint64_t last = ~0ull;
        for (int rank = 0; rank < want; ++rank) {
          uint64_t key = 0;
          for (int64_t i = threadIdx.x; i < r.n; i += NT) {
            const uint64_t q = key_of(to_f32(r.l[i]), first + (int)i);
            if (q < last && q > key) key = q;
          }
          last = over_row<NT>(key, kl, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
          if (threadIdx.x == 0) put(rank, last);
        }
      }
      for (int rank = want + (int)threadIdx.x; rank < a.top; rank += NT) put(rank, 0);   // (of a part alone)
    }
    __syncthreads();
  }
}

// A row's results from those of its parts, in their order.
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a) {
  __shared__ uint64_t keys[1024];   // parts * top at most
  __shared__ int count;
  __shared__ int ranks[256];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    // every wave by itself: a part a lane
    const int n = a.parts * a.top, lane = threadIdx.x & 63;
    const uint64_t* given = a.part_keys + row * n;
    uint64_t key[4], least = a.top && lane < a.parts ? given[lane * a.top + a.top - 1] : 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) key[q] = q * 256 + (int)threadIdx.x < n ? given[q * 256 + threadIdx.x] : 0;
    if (threadIdx.x == 0) count = 0;
    const float* sums = a.part_sums + (row * a.parts + (lane < a.parts ? lane : 0)) * 3;
    float mi = sums[0], si = sums[1], ei = sums[2];
    if (lane >= a.parts) {
      mi = -kInf;
      si = ei = 0.f;
    }
    float m = mi;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    const int at = __ffsll(__ballot(mi == m)) - 1;
    float s = si, e = ei;
    if (lane != at) {
      // (a part of -inf alone has nothing to give; of a NaN alone, a NaN)
      const float d = fmaxf(mi - m, -1000.f), w = mi == -kInf ? 0.f : exp_of(d);
      s = w * (1.f + si) + (si != si ? si : 0.f);
      e = w * (ei - d * (1.f + si));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      s += __shfl_xor(s, o);
      e += __shfl_xor(e, o);
    }
    const bool none = m == -kInf && s == 0.f;
    if (m == kInf) s = __builtin_nanf("");
    const float ls = log1pf(s);
    if (threadIdx.x == 0) put_row(a, row, m, ls, ls + e / (1.f + s), none);
    if (a.top) {
      // a part whose last key is the largest of the parts' last ones has `top` that reach it: few others do
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t k = __shfl_xor(least, o);
        least = k > least ? k : least;
      }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (key[q] && key[q] >= least) keys[atomicAdd(&count, 1)] = key[q];
      __syncthreads();
      rank_keys<256>(keys, count, a.top, ranks, [&](int rank, uint64_t k) {
        a.ids[row * a.top + rank] = index_of(k);
        a.tops[row * a.top + rank] = none ? -kInf : (logit_of(k) - m) - ls;
      });
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

template <typename T, int NT>
hipError_t go(const LogprobArgs& a, hipStream_t st) {
  const int64_t blocks = a.rows * a.parts;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), block(NT);
  if (a.top) hipLaunchKernelGGL((logprob_kernel<T, NT, true, true>), grid, block, 0, st, a);
  else if (a.ent) hipLaunchKernelGGL((logprob_kernel<T, NT, true, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((logprob_kernel<T, NT, false, false>), grid, block, 0, st, a);
  if (a.parts > 1)
    hipLaunchKernelGGL(logprob_join_kernel, dim3((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20)), dim3(256), 0,
                       st, a);
  return hipGetLastError();
}

// A wave for a row that it goes through in two groups, else 256 threads.
template <typename T>
hipError_t pick(const LogprobArgs& a, hipStream_t st) {
  return a.per <= 64 * 4 * Piece<T>::N ? go<T, 64>(a, st) : go<T, 256>(a, st);
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

// Few rows are cut into parts that a workgroup holds in registers, at most 64, which is what a wave joins (with
// alternatives, at most 1024 of these a row).  64 rows of 50304 bfloat16 with 20 alternatives
// take 18 us so, 26 in parts twice as long.
void plan_logprobs(LogprobArgs& a, int dtype) {
  const int group = 2 * 256 * (dtype == DLA_BF16 ? 8 : 4);
  int64_t parts = a.rows < 512 ? (1024 + a.rows) / (a.rows + 1) : 1;
  if (parts > (a.V + group - 1) / group) parts = (a.V + group - 1) / group;
  const int most = a.top > 16 ? 1024 / a.top : 64;
  if (parts > most) parts = most;
  if (parts < 1) parts = 1;
  a.per = (int)(((a.V + parts - 1) / parts + 7) / 8 * 8);
  a.parts = (a.V + a.per - 1) / a.per;
}

hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t st) {
  return dtype == DLA_BF16 ? pick<bf16_t>(a, st) : pick<float>(a, st);
}

hipError_t launch_logprobs_backward(const LogprobArgs& a, int dtype, hipStream_t st) {
  return dtype == DLA_BF16 ? back<bf16_t>(a, st) : back<float>(a, st);
}

}  // namespace dla
