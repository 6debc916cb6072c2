// Sums and maxima over the 64 lanes of a wave through the data-parallel-primitive moves: four shifts inside each row of 16 lanes, then
// two broadcasts of a row's last lane into the rows after it.  The result stands in lane 63 and is read from there into every lane.
// A step is one instruction of a few cycles, where an exchange through the LDS crossbar takes some fifty.  The order of the additions is fixed.
#pragma once

#include <hip/hip_runtime.h>

namespace mi355conv {

// Lane l's value from the lane that the control word names, `otherwise` where there is none or the row is masked off.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_move(int otherwise, int v) {
  return __builtin_amdgcn_update_dpp(otherwise, v, CTRL, ROWS, 0xF, false);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_move(float otherwise, float v) {
  return __builtin_bit_cast(float, dpp_move<CTRL, ROWS>(__builtin_bit_cast(int, otherwise), __builtin_bit_cast(int, v)));
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_move(double otherwise, double v) {
  const uint64_t o = __builtin_bit_cast(uint64_t, otherwise), u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)dpp_move<CTRL, ROWS>((int)(uint32_t)o, (int)(uint32_t)u);
  const uint32_t hi = (uint32_t)dpp_move<CTRL, ROWS>((int)(uint32_t)(o >> 32), (int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ float read_lane(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

__device__ __forceinline__ uint64_t read_lane(uint64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ double read_lane(double v, int lane) { return __builtin_bit_cast(double, read_lane(__builtin_bit_cast(uint64_t, v), lane)); }

template <typename T, class Op>
__device__ __forceinline__ T wave_reduce(T v, T neutral, Op op) {
  v = op(v, dpp_move<0x111, 0xF>(neutral, v));  // from 1, 2, 4, 8 lanes before
  v = op(v, dpp_move<0x112, 0xF>(neutral, v));
  v = op(v, dpp_move<0x114, 0xF>(neutral, v));
  v = op(v, dpp_move<0x118, 0xF>(neutral, v));
  v = op(v, dpp_move<0x142, 0xA>(neutral, v));  // rows 0 and 2 into rows 1 and 3
  v = op(v, dpp_move<0x143, 0xC>(neutral, v));  // rows 0 and 1 into rows 2 and 3
  return read_lane(v, 63);
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
  return wave_reduce(v, (T)0, [](T a, T b) { return a + b; });
}

__device__ __forceinline__ float wave_most(float v) {
  return wave_reduce(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}

// The maximum over each group of N neighbouring lanes (N up to 16), in every lane of the group.
template <int N>
__device__ __forceinline__ float group_most(float v) {
  if (N >= 2) v = fmaxf(v, dpp_move<0xB1, 0xF>(v, v));   // lane ^ 1
  if (N >= 4) v = fmaxf(v, dpp_move<0x4E, 0xF>(v, v));   // lane ^ 2
  if (N >= 8) v = fmaxf(v, dpp_move<0x141, 0xF>(v, v));  // 7 - lane % 8
  if (N >= 16) v = fmaxf(v, dpp_move<0x140, 0xF>(v, v)); // 15 - lane % 16
  return v;
}

}  // namespace mi355conv
