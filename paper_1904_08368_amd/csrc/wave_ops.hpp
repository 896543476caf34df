// Sums over the 64 lanes of a wave, in a fixed order, the same bits in every lane.
#pragma once
#include "attn_common.hpp"

namespace relay {

template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// neighbours, pairs of neighbours, halves of eight and of sixteen mirrored; then the sixteens
__device__ __forceinline__ float wave_sum(float v) {
  v += lane_moved<0xB1>(v);
  v += lane_moved<0x4E>(v);
  v += lane_moved<0x141>(v);
  v += lane_moved<0x140>(v);
  return sum_quarters(v);
}

}  // namespace relay
