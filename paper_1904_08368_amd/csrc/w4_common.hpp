// What the kernels of 4-bit weights share: codes as operands of the matrix cores, and a sum formed code by code.
#pragma once
#include "attention.hpp"

namespace relay {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

template <typename T> struct W4Type;
template <> struct W4Type<_Float16> {
  typedef halfx8 vec;
  // 16 + code: bits 6..9 of the half 0x4C00
  static constexpr unsigned kMask = 0x03c003c0u, kBase = 0x4c004c00u, kOne = 0x3c003c00u;
  static constexpr int kAt = 6;
  static __device__ __forceinline__ floatx4 mfma(vec a, vec b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct W4Type<__bf16> {
  typedef bfx8 vec;
  // 16 + code: bits 3..6 of 0x4180
  static constexpr unsigned kMask = 0x00780078u, kBase = 0x41804180u, kOne = 0x3f803f80u;
  static constexpr int kAt = 3;
  static __device__ __forceinline__ floatx4 mfma(vec a, vec b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// Eight codes of a word -> the eight numbers 16 + code.  The packed word is turned left by kAt bits, so that pair j comes to its place by a turn
// right of 4 j.  Mask and base are kept in registers: of the literals they are, the compiler makes two instructions of each and-or, and
// this is half of all that a byte of codes costs.
template <typename T>
struct Widen {
  unsigned mask, base;
  __device__ Widen() : mask(W4Type<T>::kMask), base(W4Type<T>::kBase) { asm("" : "+v"(mask), "+v"(base)); }
  __device__ __forceinline__ typename W4Type<T>::vec operator()(unsigned w) const {
    const uintx4 r = {(w & mask) | base, (__builtin_rotateright32(w, 4) & mask) | base, (__builtin_rotateright32(w, 8) & mask) | base,
                      (__builtin_rotateright32(w, 12) & mask) | base};
    return __builtin_bit_cast(typename W4Type<T>::vec, r);
  }
};

// One sum from the packed weights themselves, code by code: unit j against a row x of k numbers.
template <typename T>
__device__ __forceinline__ float sum_by_weights(const void* packed, const W4Layout& l, int k, int group, int zeros, const T* x, int j) {
  const unsigned char* const base = static_cast<const unsigned char*>(packed);
  const unsigned* const codes = reinterpret_cast<const unsigned*>(base) + ((size_t)(j >> 4) * l.chunks * 64 + (j & 15)) * 4;
  const size_t params = (size_t)(j >> 4) * l.groups * 16 + (j & 15);
  float sum = 0.f;
  for (int g = 0; g < l.groups && sum == sum; ++g) {
    const float scale = (float)reinterpret_cast<const T*>(base + l.scales_at)[params + (size_t)g * 16];
    const int zero = zeros ? base[l.zeros_at + params + (size_t)g * 16] - 16 : 8, end = min(k - g * group, group) + g * group;
    for (int i = g * group; i < end; i += 8) {   // (a word of the packed order: chunk i / 128, step of 32, quarter of 8)
      const unsigned w = __builtin_rotateright32(codes[((size_t)(i >> 7) * 64 + 16 * (i >> 3 & 3)) * 4 + (i >> 5 & 3)], W4Type<T>::kAt);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)x[i + e], (float)((int)(w >> (16 * (e & 1) + 4 * (e >> 1)) & 15u) - zero) * scale, sum);
    }
  }
  return sum;
}
__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) < __builtin_inff(); }
__device__ __forceinline__ bool is_finite(floatx4 v) { return is_finite(v[0]) && is_finite(v[1]) && is_finite(v[2]) && is_finite(v[3]); }

}  // namespace relay
