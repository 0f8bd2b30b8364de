// Exchanges between the lanes of a wave without LDS, and sums over them.
#pragma once

#include "ra_device.h"

namespace ra {

// Another lane's value: of the lane that the data path's pattern names (a few cycles, where an
// exchange through LDS takes over a hundred), 0 where it names none or the row of 16 lanes is
// not in kRows; and of one lane for all.
template <int kPattern, int kRows, typename V>
__device__ __forceinline__ V lane_pattern(V x) {
  if constexpr (sizeof(V) == 8) {
    const u32x2 w = __builtin_bit_cast(u32x2, x);
    u32x2 y;
    y[0] = lane_pattern<kPattern, kRows>(w[0]);
    y[1] = lane_pattern<kPattern, kRows>(w[1]);
    return __builtin_bit_cast(V, y);
  } else {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kPattern,
                                                             kRows, 0xf, false));
  }
}
template <typename V>
__device__ __forceinline__ V of_lane(V x, int lane) {
  if constexpr (sizeof(V) == 8) {
    const u32x2 w = __builtin_bit_cast(u32x2, x);
    u32x2 y;
    y[0] = of_lane(w[0], lane);
    y[1] = of_lane(w[1], lane);
    return __builtin_bit_cast(V, y);
  } else {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
  }
}
constexpr int kSwapOnes = 0xb1, kSwapTwos = 0x4e, kMirrorHalf = 0x141, kMirrorRow = 0x140;
constexpr int kShiftRow = 0x110, kLast15 = 0x142, kLast31 = 0x143;

// Sums up to and with this lane.
template <typename V>
__device__ __forceinline__ V wave_sums(V x) {
  x += lane_pattern<kShiftRow + 1, 0xf>(x);
  x += lane_pattern<kShiftRow + 2, 0xf>(x);
  x += lane_pattern<kShiftRow + 4, 0xf>(x);
  x += lane_pattern<kShiftRow + 8, 0xf>(x);
  x += lane_pattern<kLast15, 0xa>(x);
  x += lane_pattern<kLast31, 0xc>(x);
  return x;
}

}  // namespace ra
