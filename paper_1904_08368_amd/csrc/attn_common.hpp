// What the attention kernels share: operand types of the matrix instructions, lane exchanges, the view of a sequence, masked blocks.
//
// Both kernels compute the scores transposed, S^T = K Q^T, and the output transposed, O^T = V^T P^T, with 16 x 16 or 32 x 32 results whose columns
// are query rows.  A lane then holds scores of one query row, and the probabilities it makes of them are, without an exchange between
// lanes, the B operand of the second product: which key stands in which place of a reduction does not matter as long as V^T, read from LDS
// through the transposing load, has the same order.
#pragma once
#include "attention.hpp"

namespace relay {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

template <typename T> struct Mma;
template <> struct Mma<_Float16> {
  typedef halfx8 vec;
  typedef _Float16 pair __attribute__((ext_vector_type(2)));
  static constexpr unsigned kExp = 0x7c007c00u;   // exponent bits of two elements
  // Probabilities are taken this power of two larger (bf16 reaches as far down as fp32 and needs none), so that fp16 still holds those 2^-22 of the largest to
  // its full precision in the kernel for few rows, 2^-18 of the reference in the other, where one may be up to 2^8 by itself.  No further: scores of 10^8 leave an exponent that is
  // off by some units, and fp16 ends at 2^16.
  static constexpr float kShiftRows = 8.f, kShiftTiles = 4.f;
  // c + the two elements of a word.  (The instruction does not round to nearest: for the few words of a step, not for a sum over all of them.)
  static __device__ __forceinline__ float add2(unsigned w, float c) { return __builtin_amdgcn_fdot2(__builtin_bit_cast(pair, w), (pair){1, 1}, c, false); }
  static __device__ __forceinline__ floatx4 mfma16(vec a, vec b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ floatx16 mfma32(vec a, vec b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<__bf16> {
  typedef bfx8 vec;
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  static constexpr unsigned kExp = 0x7f807f80u;
  static constexpr float kShiftRows = 0.f, kShiftTiles = 0.f;
  static __device__ __forceinline__ float add2(unsigned w, float c) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, w), __builtin_bit_cast(pair, 0x3f803f80u), c, false); }
  static __device__ __forceinline__ floatx4 mfma16(vec a, vec b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ floatx16 mfma32(vec a, vec b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// two fp32 numbers rounded to nearest into one word
template <typename T>
__device__ __forceinline__ unsigned pack2(float a, float b) {
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((floatx2){a, b}, typename Mma<T>::pair));
}

// The values of lanes l and l ^ 32 (l ^ 16).
struct LanePair { float a, b; };
__device__ __forceinline__ LanePair pair_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned r0 = r[0], r1 = r[1];   // (a bit cast of a vector's element itself reads element 0)
  return {__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)};
}
__device__ __forceinline__ LanePair pair_quarters(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned r0 = r[0], r1 = r[1];
  return {__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)};
}
// maximum and sum over the lanes l, l ^ 32 and over l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float max_halves(float v) { const LanePair p = pair_halves(v); return fmaxf(p.a, p.b); }
__device__ __forceinline__ float sum_halves(float v) { const LanePair p = pair_halves(v); return p.a + p.b; }
__device__ __forceinline__ float max_quarters(float v) { const LanePair p = pair_quarters(v); return max_halves(fmaxf(p.a, p.b)); }
__device__ __forceinline__ float sum_quarters(float v) { const LanePair p = pair_quarters(v); return sum_halves(p.a + p.b); }

// 2^x (results below 2^-126 flush to zero: beside a largest probability of 1 they do not count)
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kNegInf = -__builtin_inff();

// four 16-bit elements of each of 16 columns, one column to a lane: p is this lane's quarter of a row (4 lanes to a row of 16 elements)
__device__ __forceinline__ uintx2 lds_transposed(const void* p) {
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (__attribute__((address_space(3))) shortx4*)(uintptr_t)(const __attribute__((address_space(3))) void*)p));
}

// does a word hold an infinity or a NaN in either half?
template <typename T>
__device__ __forceinline__ bool not_finite(unsigned w) {
  constexpr unsigned lo = Mma<T>::kExp & 0xffffu, hi = Mma<T>::kExp & 0xffff0000u;
  return (w & lo) == lo || (w & hi) == hi;
}
// ... replaced by zeros
template <typename T>
__device__ __forceinline__ unsigned only_finite(unsigned w) {
  constexpr unsigned lo = Mma<T>::kExp & 0xffffu, hi = Mma<T>::kExp & 0xffff0000u;
  if ((w & lo) == lo) w &= 0xffff0000u;
  if ((w & hi) == hi) w &= 0x0000ffffu;
  return w;
}

// Arrival counters lie 64 bytes apart in front of the workspace, in a region of their own that is the same for every call.
constexpr int kCounters = 1024;
constexpr size_t kCounterBytes = (size_t)kCounters * 64;

// One sequence as a workgroup sees it.  Its tokens' positions go by its true length; keys past the table's pages, or past the bound that the launch
// was sized by, are not there to be seen.
struct Seq {
  int start, nq, kv;   // first row of q; new tokens; keys that can be read
  int before;          // keys ahead of the first new token: its position
  __device__ Seq(const AttnArgs& a, int b) {
    start = a.q_starts[b];
    nq = a.q_starts[b + 1] - start;
    const int length = max(a.kv_lens[b], 0);
    kv = min(length, a.max_kv_len);
    before = length - nq;
  }
  // keys that token i sees: first, last (none if last < first).  (A window of up to 2^31 - 1 behind a token ahead of the first key: 64 bits.)
  __device__ int first(const AttnArgs& a, int i) const { return a.window > 0 ? (int)min((long)kv, max(0L, (long)before + i - a.window + 1)) : 0; }
  __device__ int last(const AttnArgs& a, int i) const { return a.causal ? min(kv - 1, before + i) : kv - 1; }
};

}  // namespace relay
