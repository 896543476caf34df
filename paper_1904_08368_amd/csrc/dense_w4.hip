// Dense with 4-bit weights and group scales:  y[m,j] = sum_g scale[j,g] sum_{i in g} x[m,i] (code[j,i] - zero[j,g])  and its fused tail.
//
// Codes enter the matrix cores as the exact 16-bit numbers 16 + code: the four bits are moved to the top of the
// mantissa of 16.0, one shift and one and-or for two of them.  With S = sum_{i in g} x[m,i], which a product with ones gives,
//   sum x (code - zero) = sum x (16 + code) - (16 + zero) S
// so the weights are never rounded and a group's scale multiplies an fp32 sum.  The offset of 16 costs the sums three bits of fp32 at most.
//
// Few rows of x: bound by the codes' bytes.  The waves of a workgroup share 16 units' rows out among them along the reduction, each
// streams its part straight into the A operands (the packed order), and they add up through LDS.
#include "attention.hpp"

namespace relay {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
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

// eight codes of a word -> the eight numbers 16 + code
template <typename T>
__device__ __forceinline__ typename W4Type<T>::vec widen(unsigned w) {
  typedef W4Type<T> C;
  uintx4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int sh = C::kAt - 4 * j;
    r[j] = ((sh >= 0 ? w << (sh > 0 ? sh : 0) : w >> (sh < 0 ? -sh : 0)) & C::kMask) | C::kBase;
  }
  return __builtin_bit_cast(typename C::vec, r);
}

// the tail of one output
template <typename T>
__device__ __forceinline__ void finish(const W4Args& a, int m, int j, float v) {
  if (a.bias) v += a.bias[j];
  if (a.res) v += (float)static_cast<const T*>(a.res)[(long)m * a.y_stride + j];
  if (a.relu) v = v > 0.f ? v : 0.f;
  static_cast<T*>(a.y)[(long)m * a.y_stride + j] = (T)v;
}

template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void w4_rows_kernel(const W4Args a, const W4Layout l) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  __shared__ floatx4 part[WAVES][64];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int tile = (int)blockIdx.x, m0 = (int)blockIdx.y * 16;
  const int g = lane >> 4, col = lane & 15;
  const int row = min(m0 + col, a.m - 1);   // (columns beyond m repeat the last row and are not stored)
  const T* x = static_cast<const T*>(a.x) + (long)row * a.x_stride + 8 * g;
  const unsigned char* base = static_cast<const unsigned char*>(a.packed);
  const uintx4* w = reinterpret_cast<const uintx4*>(base) + (size_t)tile * l.chunks * 64 + lane;
  // this lane's sums belong to units 4 g .. 4 g + 3 of the tile and to row `col`
  const T* scales = reinterpret_cast<const T*>(base + l.scales_at) + (size_t)tile * l.groups * 16 + 4 * g;
  const unsigned char* zeros = base + l.zeros_at + (size_t)tile * l.groups * 16 + 4 * g;
  const int steps = (a.k + 31) / 32, per_group = a.group / 32;
  // a wave takes whole groups
  const int first = l.groups * wave / WAVES, last = l.groups * (wave + 1) / WAVES;
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  floatx4 sum = {0, 0, 0, 0};
  for (int gr = first; gr < last; ++gr) {
    floatx4 acc = {0, 0, 0, 0}, xs = {0, 0, 0, 0};
    const int s1 = min((gr + 1) * per_group, steps);
    for (int s = gr * per_group; s < s1; ++s) {
      const unsigned code = w[(size_t)(s >> 2) * 64][s & 3];
      vec xv = __builtin_bit_cast(vec, (uintx4){0, 0, 0, 0});
      if (s * 32 + 8 * g < a.k) xv = *reinterpret_cast<const vec*>(x + s * 32);
      acc = C::mfma(widen<T>(code), xv, acc);
      xs = C::mfma(ones, xv, xs);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float z = 16.f + (a.zeros ? (float)zeros[gr * 16 + i] : 8.f);
      sum[i] = fmaf((float)scales[gr * 16 + i], fmaf(-z, xs[i], acc[i]), sum[i]);
    }
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int u = 1; u < WAVES; ++u) sum += part[u][lane];
  if (m0 + col >= a.m) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = tile * 16 + 4 * g + i;
    if (j < a.n) finish<T>(a, m0 + col, j, sum[i]);
  }
}

// a thread packs one word: eight codes, or one scale, or one zero point
__global__ __launch_bounds__(256) void w4_pack_kernel(int n, int k, int zeros, W4Layout l, const uint8_t* codes, const uint16_t* scales,
                                                      const uint8_t* zps, unsigned char* out) {
  const size_t words = (size_t)l.tiles * l.chunks * 256, params = (size_t)l.tiles * l.groups * 16;
  for (size_t t = (size_t)blockIdx.x * 256 + threadIdx.x; t < words + params; t += (size_t)gridDim.x * 256) {
    if (t < words) {
      const int s = (int)(t & 3), lane = (int)(t >> 2) & 63;
      const size_t block = t >> 8;
      const int tile = (int)(block / l.chunks), chunk = (int)(block % l.chunks);
      const int j = tile * 16 + (lane & 15), i = chunk * 128 + s * 32 + (lane >> 4) * 8;
      unsigned w = 0;
      if (j < n && i < k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned b = codes[(size_t)j * (k / 2) + i / 2 + e];
          w |= (b & 15u) << (4 * e) | (b >> 4) << (16 + 4 * e);
        }
      }
      reinterpret_cast<unsigned*>(out)[t] = w;
    } else {
      const size_t u = t - words;
      const int j = (int)(u / ((size_t)l.groups * 16)) * 16 + (int)(u & 15), gr = (int)(u / 16 % l.groups);
      reinterpret_cast<uint16_t*>(out + l.scales_at)[u] = j < n ? scales[(size_t)j * l.groups + gr] : (uint16_t)0;
      if (zeros) (out + l.zeros_at)[u] = j < n ? zps[(size_t)j * l.groups + gr] : (uint8_t)0;
    }
  }
}

}  // namespace

hipError_t launch_w4_pack(const W4Args& a, const uint8_t* codes, const void* scales, const uint8_t* zeros, void* packed, hipStream_t st) {
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.zeros != 0);
  const size_t items = (size_t)l.tiles * l.chunks * 256 + (size_t)l.tiles * l.groups * 16;
  const unsigned grid = (unsigned)((items + 255) / 256 < 65536 ? (items + 255) / 256 : 65536);
  hipLaunchKernelGGL(w4_pack_kernel, dim3(grid), dim3(256), 0, st, a.n, a.k, a.zeros, l, codes, static_cast<const uint16_t*>(scales), zeros,
                     static_cast<unsigned char*>(packed));
  return hipGetLastError();
}

bool w4_fits(const W4Args& a) { return a.m <= 16 * 65535; }

hipError_t launch_w4(const W4Args& a, int dtype, hipStream_t st) {
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.zeros != 0);
  const dim3 grid((unsigned)l.tiles, (unsigned)((a.m + 15) / 16));
  if (dtype == T_F16) hipLaunchKernelGGL((w4_rows_kernel<_Float16, 8>), grid, dim3(512), 0, st, a, l);
  else hipLaunchKernelGGL((w4_rows_kernel<__bf16, 8>), grid, dim3(512), 0, st, a, l);
  return hipGetLastError();
}

}  // namespace relay
