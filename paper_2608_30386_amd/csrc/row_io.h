// Rows of bf16, fp16 or fp32 elements in vectors that need no alignment beyond their element's: rows of
// an odd width start anywhere, and the hardware takes wide accesses at any address.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dasc/ops.h"

namespace dasc {

struct bf16_t { uint16_t bits; };
struct f16_t { _Float16 x; };

__device__ inline float widen(bf16_t v) { return __uint_as_float(uint32_t(v.bits) << 16); }
__device__ inline float widen(f16_t v) { return float(v.x); }
__device__ inline float widen(float v) { return v; }
__device__ inline void narrow(float x, bf16_t& v) { v.bits = __builtin_bit_cast(uint16_t, __bf16(x)); }
__device__ inline void narrow(float x, f16_t& v) { v.x = _Float16(x); }
__device__ inline void narrow(float x, float& v) { v = x; }

template <typename T, int N>
struct __attribute__((packed, aligned(alignof(T)))) Vec { T e[N]; };

// Elements [c, c + N) of a row of n, those beyond its end as zero
template <int N, typename T>
__device__ inline void load_vec(const T* row, int c, int n, float* x) {
  if (c + N <= n) {
    const Vec<T, N> v = *reinterpret_cast<const Vec<T, N>*>(row + c);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = widen(v.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.0f;
    if (c < n) {
#pragma unroll
      for (int i = 0; i < N - 1; ++i)
        if (c + i < n) x[i] = widen(row[c + i]);
    }
  }
}

template <int N, typename T>
__device__ inline void store_vec(T* row, int c, int n, const float* x) {
  if (c + N <= n) {
    Vec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) narrow(x[i], v.e[i]);
    *reinterpret_cast<Vec<T, N>*>(row + c) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (c + i < n) narrow(x[i], row[c + i]);
  }
}

}  // namespace dasc
