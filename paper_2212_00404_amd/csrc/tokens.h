// Shared by the kernels over tokens (rotate, join, attend): element types,
// their conversion to and from fp32, and reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "dconv.h"

namespace dconv {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

inline int element_size(int dtype) {
  return dtype == DCONV_F32 ? 4 : dtype == DCONV_F16 || dtype == DCONV_BF16 ? 2 : 0;
}

// Conversions round to nearest even; fp16 values past 65504 become infinities.
template <class T>
__device__ __forceinline__ float to_f32(T x) {
  return static_cast<float>(x);
}
template <class T>
__device__ __forceinline__ T from_f32(float x) {
  return static_cast<T>(x);
}

// Sum / maximum over groups of N lanes (N a power of two up to 64): every lane
// gets the result, and all lanes add in the same order.
template <int N>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
template <int N>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

}  // namespace dconv
