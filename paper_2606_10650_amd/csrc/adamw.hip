// One AdamW step over many tensors: one launch per kTensors of them, whose descriptions
// travel as the kernel's argument, so that no table lives on the device and the call can be
// recorded.  A workgroup takes kChunk elements of one tensor, a wave 256 at a time: four
// consecutive ones a lane, and with 8-bit states one block, whose scales it forms with lane
// moves.  Every byte is read and written once; they bound it: 134M bfloat16 parameters with
// float32 masters 736 us for 3.8 GB, 5.1 TB/s, a large copy's rate; with 8-bit states 463 us
// for 2.1 GB, 4.6 TB/s, where the roots, hashes and conversions show.
//
// 8-bit states are codes of m and of r = sqrt(v) (4 exponent and 3 mantissa bits) times a
// float32 scale per 256 elements, the block's largest magnitude / 448.  The root halves the
// exponents' range: 2^-17 of the block's largest r still has a code.  An r above zero never
// gets the code zero: its m may not have, and m / eps would be a step without bound.  The
// moving averages move by 1 - beta of their distance in a step, for v a thousandth, where
// neighbouring codes are 6 to 12% apart: rounded to nearest they would stand still, so a
// call may give a seed, and values are rounded to either neighbour with the probability
// that makes the average right.
#include "adamw.h"

namespace dla {
namespace {

constexpr int kTensors = 40;
constexpr int kChunk = 4096;
constexpr int kBlock = 256;
constexpr uint64_t kGroups = 0xFFFFFFFFu / 256;   // a launch has fewer than 2^32 threads
static_assert(kAdamWMost / kChunk <= kGroups, "a tensor fits one launch");

struct Table {
  dla_adamw_tensor t[kTensors];
  uint32_t first[kTensors + 1];   // a tensor's first workgroup; from n on, the grid's size
  uint32_t number;                // the first tensor's number in the call
  AdamWScalars s;
};

template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, bool wide, float (&x)[4]) {
  if (wide && n >= 4) {
    if constexpr (sizeof(T) == 2) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      x[0] = __uint_as_float(u.x << 16);
      x[1] = __uint_as_float(u.x & 0xFFFF0000u);
      x[2] = __uint_as_float(u.y << 16);
      x[3] = __uint_as_float(u.y & 0xFFFF0000u);
    } else {
      const float4 u = *reinterpret_cast<const float4*>(p);
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void put4(T* p, int n, bool wide, const float (&x)[4]) {
  if constexpr (sizeof(T) == 2) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    if (wide && n >= 4) {
      bf16x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (__bf16)x[i];
      *reinterpret_cast<bf16x4*>(p) = y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) reinterpret_cast<__bf16*>(p)[i] = (__bf16)x[i];
    }
  } else {
    if (wide && n >= 4) {
      *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) p[i] = x[i];
    }
  }
}
__device__ __forceinline__ void load_codes(const uint8_t* p, int n, bool wide, float (&x)[4]) {
  uint32_t u = 0;
  if (wide && n >= 4) {
    u = *reinterpret_cast<const uint32_t*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) u |= (uint32_t)p[i] << (8 * i);
  }
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}
__device__ __forceinline__ void put_codes(uint8_t* p, int n, bool wide, const float (&x)[4]) {
  uint32_t u = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  u = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], u, true);
  if (wide && n >= 4) {
    *reinterpret_cast<uint32_t*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = (uint8_t)(u >> (8 * i));
  }
}

// 32 bits from an element's index, its tensor's number and the call's seed: two rounds of
// multiplying and folding.
__device__ __forceinline__ uint32_t random_bits(uint32_t index, uint32_t number, uint32_t seed) {
  uint32_t h = (index + 0x9E3779B9u * (number + 1)) ^ seed;
  h *= 0x2545F491u;
  h ^= h >> 16;
  h *= 0x9E3779B1u;
  return h ^ (h >> 15);
}

// x, of magnitude 448 at most up to rounding, as a number that has a code.  u in [0, 1):
// up if the part between two codes and u come to one; u < 0: to the nearest, by the
// conversion that follows.
__device__ __forceinline__ float to_code(float x, float u) {
  float y = fabsf(x);
  if (u >= 0.f) {
    const uint32_t e = max((__float_as_uint(y) >> 23) & 255u, 121u);   // 2^-6 and below: one spacing
    y = floorf(y * __uint_as_float((257u - e) << 23) + u) * __uint_as_float((e - 3u) << 23);
  }
  y = y > 448.f ? 448.f : y;
  return copysignf(y, x);
}

__device__ __forceinline__ float block_top(const float (&x)[4]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y = fabsf(x[i]);
    top = y > top || y != y ? y : top;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float y = __shfl_xor(top, o);
    top = y > top || y != y ? y : top;
  }
  return top;
}

__device__ __forceinline__ float lane_value(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

constexpr float kLeastTop = 1e-30f;   // a block whose largest value is below this is all zero

template <typename Tp, typename Tg, bool F8>
__global__ __launch_bounds__(256) void adamw_kernel(Table tab) {
  const AdamWScalars& s = tab.s;
  float scale = 1.f;
  if (s.grad_scale) {
    scale = *s.grad_scale;
    if (!(fabsf(scale) <= 0x1.fffffep127f)) return;
  }
  int k = 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    if (k + o < kTensors && tab.first[k + o] <= blockIdx.x) k += o;
  const dla_adamw_tensor& t = tab.t[k];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t begin = (int64_t)(blockIdx.x - tab.first[k]) * kChunk;
  Tp* param = static_cast<Tp*>(t.param);
  const Tg* grad = static_cast<const Tg*>(t.grad);
  // a lane's elements start at multiples of four, so the bases decide
  const uintptr_t f32 = (uintptr_t)t.master | (F8 ? 0 : (uintptr_t)t.m | (uintptr_t)t.v);
  const bool wide = !(f32 & 15) && !((uintptr_t)param & (4 * sizeof(Tp) - 1)) &&
                    !((uintptr_t)grad & (4 * sizeof(Tg) - 1)) &&
                    !(F8 && (((uintptr_t)t.m | (uintptr_t)t.v) & 3));
  const float keep = 1.f - s.lr * t.weight_decay;
#pragma unroll
  for (int it = 0; it < kChunk / 1024; ++it) {
    const int64_t b0 = begin + (it * 4 + wave) * kBlock, i = b0 + 4 * lane;
    if (b0 >= t.n) break;   // the whole wave's elements
    const int64_t left = t.n - i;
    const int n = left < 0 ? 0 : (left > 4 ? 4 : (int)left);
    float g[4], p[4], m[4], v[4];
    load4(grad + i, n, wide, g);
    if (t.master) load4(t.master + i, n, wide, p);
    else load4(param + i, n, wide, p);
    const int64_t blk = b0 / kBlock;
    if constexpr (F8) {
      load_codes(static_cast<const uint8_t*>(t.m) + i, n, wide, m);
      load_codes(static_cast<const uint8_t*>(t.v) + i, n, wide, v);
      const float ms = t.m_scale[blk], vs = t.v_scale[blk];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] *= ms;
        v[j] *= vs;
        v[j] *= v[j];
      }
    } else {
      load4(static_cast<const float*>(t.m) + i, n, wide, m);
      load4(static_cast<const float*>(t.v) + i, n, wide, v);
    }
    float root[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // every operation rounded, none contracted: a last bit can decide a code, and a code
      // decides the next step, so states are to follow from dla_train.h's lines alone
#pragma clang fp contract(off)
      g[j] *= scale;
      m[j] = s.beta1 * m[j] + s.rest1 * g[j];
      v[j] = s.beta2 * v[j] + s.rest2 * g[j] * g[j];
      root[j] = sqrtf(v[j]);
      p[j] = p[j] * keep - s.step_size * m[j] / (root[j] * s.root2 + s.eps);
    }
    if (t.master) put4(t.master + i, n, wide, p);
    put4(param + i, n, wide, p);
    if constexpr (F8) {
      const float mt = block_top(m), vt = block_top(root);
      // both kinds by one division: m's in lane 0, the root's in lane 1
      const float top = lane & 1 ? vt : mt;
      const bool some = top > kLeastTop;
      const float none = top <= kLeastTop ? 0.f : top;   // (a NaN stays one)
      const float inv = some ? 1.f / top * 448.f : none;
      const float mi = lane_value(inv, 0), vi = lane_value(inv, 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float um = -1.f, uv = -1.f;
        if (s.seed) {
          const uint32_t r = random_bits((uint32_t)(i + j), tab.number + k, s.seed);
          um = (float)(r >> 16) * (1.f / 65536.f);
          uv = (float)(r & 0xFFFFu) * (1.f / 65536.f);
        }
        m[j] = to_code(m[j] * mi, um);
        const bool least = root[j] > 0.f && vi > 0.f;
        v[j] = to_code(root[j] * vi, uv);
        if (least && v[j] < 0.001953125f) v[j] = 0.001953125f;   // 2^-9, the least code
      }
      put_codes(static_cast<uint8_t*>(t.m) + i, n, wide, m);
      put_codes(static_cast<uint8_t*>(t.v) + i, n, wide, v);
      const float unit = some ? top * (1.f / 448.f) : none;
      if (lane == 0) t.m_scale[blk] = unit;
      if (lane == 1) t.v_scale[blk] = unit;
    } else {
      put4(static_cast<float*>(t.m) + i, n, wide, m);
      put4(static_cast<float*>(t.v) + i, n, wide, v);
    }
  }
}

template <typename Tp, typename Tg>
void go(const Table& tab, uint32_t grid, bool f8, hipStream_t st) {
  if (f8) hipLaunchKernelGGL((adamw_kernel<Tp, Tg, true>), dim3(grid), dim3(256), 0, st, tab);
  else hipLaunchKernelGGL((adamw_kernel<Tp, Tg, false>), dim3(grid), dim3(256), 0, st, tab);
}

}  // namespace

hipError_t launch_adamw(const dla_adamw_tensor* t, int n, const AdamWScalars& s, int param_dtype,
                        int grad_dtype, bool f8, hipStream_t st) {
  int i = 0;
  while (i < n) {
    Table tab;
    tab.s = s;
    tab.number = (uint32_t)i;
    uint64_t grid = 0;
    int k = 0;
    for (; k < kTensors; ++k) {
      tab.t[k] = dla_adamw_tensor{};
      tab.first[k] = (uint32_t)grid;
      if (i + k < n) {
        const uint64_t groups = (uint64_t)((t[i + k].n + kChunk - 1) / kChunk);
        if (grid + groups > kGroups) break;   // the rest goes by the next launch
        tab.t[k] = t[i + k];
        grid += groups;
      }
    }
    const int taken = k < n - i ? k : n - i;
    for (; k < kTensors; ++k) {
      tab.t[k] = dla_adamw_tensor{};
      tab.first[k] = (uint32_t)grid;
    }
    tab.first[kTensors] = (uint32_t)grid;
    // Tensors without elements have no workgroup: the search below finds the last tensor
    // whose first workgroup is not behind a given one, and that one has elements.
    if (grid) {
      if (param_dtype == DLA_BF16) {
        if (grad_dtype == DLA_BF16) go<bf16_t, bf16_t>(tab, (uint32_t)grid, f8, st);
        else go<bf16_t, float>(tab, (uint32_t)grid, f8, st);
      } else {
        if (grad_dtype == DLA_BF16) go<float, bf16_t>(tab, (uint32_t)grid, f8, st);
        else go<float, float>(tab, (uint32_t)grid, f8, st);
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    i += taken;
  }
  return hipSuccess;
}

}  // namespace dla
