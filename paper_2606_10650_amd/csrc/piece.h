// Pieces of 16 bytes of rows that may start at any element: a piece is read and written as it
// lies, whatever its alignment, with the elements from n on left out.
#pragma once
#include "dla_common.h"

namespace dla {

template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    uint32_t w[4];
  };
  // a piece as it lies, zero from element n on
  __device__ static __forceinline__ Raw raw(const T* p, int n) {
    if (n >= N) return *reinterpret_cast<const Raw*>(p);
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i < n) {
        if constexpr (sizeof(T) == 2) r.w[i >> 1] |= (uint32_t)p[i].x << (16 * (i & 1));
        else r.w[i] = __float_as_uint(p[i]);
      }
    }
    return r;
  }
  __device__ static __forceinline__ float value(const Raw& r, int i) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? r.w[i >> 1] & 0xFFFF0000u : r.w[i >> 1] << 16);
    else return __uint_as_float(r.w[i]);
  }
  __device__ static __forceinline__ void load(const T* p, int n, float (&x)[N]) {
    const Raw r = raw(p, n);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = value(r, i);
  }
  __device__ static __forceinline__ void store(T* p, int n, const float (&x)[N]) {
    if constexpr (sizeof(T) == 2) {
      if (n >= N) {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
          bf16x2 y;
          y[0] = (__bf16)x[2 * i];
          y[1] = (__bf16)x[2 * i + 1];
          r.w[i] = __builtin_bit_cast(uint32_t, y);
        }
        *reinterpret_cast<Raw*>(p) = r;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < n) reinterpret_cast<__bf16*>(p)[i] = (__bf16)x[i];
      }
    } else {
      if (n >= N) {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = __float_as_uint(x[i]);
        *reinterpret_cast<Raw*>(p) = r;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < n) p[i] = x[i];
      }
    }
  }
};

// Elements i .. i + N - 1 of an array of type T or float32 as floats, zero from element n on.
template <typename T>
__device__ __forceinline__ void load_floats(const void* p, int f32, int64_t i, int n, float (&x)[Piece<T>::N]) {
  if (sizeof(T) == 4 || f32) {
    using P = Piece<float>;
#pragma unroll
    for (int q = 0; q < Piece<T>::N; q += P::N) {
      const P::Raw r = P::raw(static_cast<const float*>(p) + i + q, n - q);
#pragma unroll
      for (int j = 0; j < P::N; ++j) x[q + j] = P::value(r, j);
    }
  } else {
    Piece<T>::load(static_cast<const T*>(p) + i, n, x);
  }
}

}  // namespace dla
