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

// The value of the lane that `CTRL` names among the 16 of a row.
template <int CTRL>
__device__ __forceinline__ float row_lane(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// f over groups of N lanes (N = 16, 32 or 64), the same bits in every lane: a
// butterfly of register moves (neighbours, pairs, the mirror images within 8 and
// 16 lanes, then exchanges of whole rows and halves), none through LDS.
template <int N, class F>
__device__ __forceinline__ float lanes_reduce(float x, F f) {
  x = f(x, row_lane<0xB1>(x));
  x = f(x, row_lane<0x4E>(x));
  x = f(x, row_lane<0x141>(x));
  x = f(x, row_lane<0x140>(x));
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (N >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return x;
}
template <int N>
__device__ __forceinline__ float lanes_sum(float x) {
  return lanes_reduce<N>(x, [](float a, float b) { return a + b; });
}
template <int N>
__device__ __forceinline__ float lanes_max(float x) {
  return lanes_reduce<N>(x, [](float a, float b) { return fmaxf(a, b); });
}

// Barrier for a hand-over through LDS: waits for this wave's LDS operations, not
// for its loads from memory.
__device__ __forceinline__ void wait_lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace dconv
