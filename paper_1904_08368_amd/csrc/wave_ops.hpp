// Sums and maxima over the 64 lanes of a wave, in a fixed order, the same bits in every lane.
#pragma once
#include <type_traits>

#include "attn_common.hpp"

namespace relay {

template <int CTRL>
__device__ __forceinline__ unsigned lane_moved(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) { return __builtin_bit_cast(float, lane_moved<CTRL>(__builtin_bit_cast(unsigned, v))); }
template <int CTRL, typename V>   // (64 bits)
__device__ __forceinline__ V lane_moved64(V v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
  return __builtin_bit_cast(V, (unsigned long long)lane_moved<CTRL>((unsigned)(u >> 32)) << 32 | lane_moved<CTRL>((unsigned)u));
}
// the values of the lane's own row of 16 and of the other of its pair, of its own half and of the other
template <typename V>
struct Pair64 { V a, b; };
template <bool HALVES, typename V>
__device__ __forceinline__ Pair64<V> pair64(V v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
  const unsigned lo = (unsigned)u, hi = (unsigned)(u >> 32);
  const auto l = HALVES ? __builtin_amdgcn_permlane32_swap(lo, lo, false, false) : __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
  const auto h = HALVES ? __builtin_amdgcn_permlane32_swap(hi, hi, false, false) : __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  const unsigned l0 = l[0], l1 = l[1], h0 = h[0], h1 = h[1];
  return {__builtin_bit_cast(V, (unsigned long long)h0 << 32 | l0), __builtin_bit_cast(V, (unsigned long long)h1 << 32 | l1)};
}

// neighbours, pairs of neighbours, halves of eight and of sixteen mirrored; then the sixteens
__device__ __forceinline__ float wave_sum(float v) {
  v += lane_moved<0xB1>(v);
  v += lane_moved<0x4E>(v);
  v += lane_moved<0x141>(v);
  v += lane_moved<0x140>(v);
  return sum_quarters(v);
}
template <typename V, typename F>   // (32 bits)
__device__ __forceinline__ V wave_fold32(V v, F f) {
  auto moved = [](V u, auto ctrl) { return __builtin_bit_cast(V, lane_moved<decltype(ctrl)::value>(__builtin_bit_cast(unsigned, u))); };
  v = f(v, moved(v, std::integral_constant<int, 0xB1>()));
  v = f(v, moved(v, std::integral_constant<int, 0x4E>()));
  v = f(v, moved(v, std::integral_constant<int, 0x141>()));
  v = f(v, moved(v, std::integral_constant<int, 0x140>()));
  const unsigned b = __builtin_bit_cast(unsigned, v);
  const auto rows = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  const unsigned r0 = rows[0], r1 = rows[1];
  v = f(__builtin_bit_cast(V, r0), __builtin_bit_cast(V, r1));
  const unsigned c = __builtin_bit_cast(unsigned, v);
  const auto halves = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  const unsigned h0 = halves[0], h1 = halves[1];
  return f(__builtin_bit_cast(V, h0), __builtin_bit_cast(V, h1));
}
template <typename V, typename F>
__device__ __forceinline__ V wave_fold64(V v, F f) {
  v = f(v, lane_moved64<0xB1>(v));
  v = f(v, lane_moved64<0x4E>(v));
  v = f(v, lane_moved64<0x141>(v));
  v = f(v, lane_moved64<0x140>(v));
  const Pair64<V> rows = pair64<false>(v);
  v = f(rows.a, rows.b);
  const Pair64<V> halves = pair64<true>(v);
  return f(halves.a, halves.b);
}
__device__ __forceinline__ double wave_sum64(double v) { return wave_fold64(v, [](double a, double b) { return a + b; }); }

}  // namespace relay
