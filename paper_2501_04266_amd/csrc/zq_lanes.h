// zq_lanes.h -- values of other lanes of a wave, and sums over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zq_device.h"

namespace zq {

template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return u2f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f2u(v), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ double from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// f over R lanes, 4 to 64, in all of them: within rows of 16 lanes through the ALUs (a shuffle
// through LDS takes ten times as long), each lane from its mirror image
template <int R, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
  v = f(v, from_lane<0xB1>(v));                      // quad_perm 1,0,3,2
  v = f(v, from_lane<0x4E>(v));                      // quad_perm 2,3,0,1
  if constexpr (R >= 8) v = f(v, from_lane<0x141>(v));   // row_half_mirror
  if constexpr (R >= 16) v = f(v, from_lane<0x140>(v));  // row_mirror
  if constexpr (R >= 32) v = f(v, __shfl_xor(v, 16));
  if constexpr (R >= 64) v = f(v, __shfl_xor(v, 32));
  return v;
}
template <int R, typename T>
__device__ __forceinline__ T lanes_sum(T v) {
  return over_lanes<R>(v, [](T a, T b) { return a + b; });
}

}  // namespace zq
