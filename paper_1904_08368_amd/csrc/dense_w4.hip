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

// Up to four rows: bound by the codes' bytes, so what else goes through the memory pipe is kept small.  The 16 columns of a matrix
// instruction are four rows by the four 32-long steps of a chunk: column 4 r + s holds row r's part of step s, one 16-byte load a
// lane for a whole chunk.  The instruction of step s gives its column its product and the others products that nobody looks at; each
// lane takes its own step's result, scaled by that step's group, and the four columns of a row meet at the end.
// W waves share the reduction out in chunks of 128; DEPTH chunks are on their way.  (Loads return in the order of their issue: a chunk's codes, x and
// scales are asked for together, or waiting for x would be waiting for the codes of chunks ahead.)
template <typename T, int W, int DEPTH>
__global__ __launch_bounds__(W * 64) void w4_few_kernel(const W4Args a, const W4Layout l, const FastDiv per_group) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  typedef T four __attribute__((ext_vector_type(4)));
  __shared__ floatx4 part[W][16];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int tile = (int)blockIdx.x, g = lane >> 4, col = lane & 15, step = col & 3, row = col >> 2;
  const unsigned char* base = static_cast<const unsigned char*>(a.packed);
  const int first = l.chunks * wave / W, last = l.chunks * (wave + 1) / W;
  const uintx4* w = reinterpret_cast<const uintx4*>(base) + (size_t)tile * l.chunks * 64 + lane;
  const T* scales = reinterpret_cast<const T*>(base + l.scales_at) + (size_t)tile * l.groups * 16 + 4 * g;
  const unsigned char* zeros = base + l.zeros_at + (size_t)tile * l.groups * 16 + 4 * g;
  const bool row_ok = row < a.m;
  const T* x = static_cast<const T*>(a.x) + (row_ok ? (long)row * a.x_stride : 0) + step * 32 + 8 * g;
  uintx4 codes[DEPTH], xv[DEPTH];
  four sc[DEPTH];
  unsigned zp[DEPTH];
  auto load = [&](int chunk, int d) {
    codes[d] = w[(size_t)chunk * 64];
    xv[d] = (uintx4){0, 0, 0, 0};
    if (row_ok && chunk * 128 + step * 32 + 8 * g < a.k) xv[d] = *reinterpret_cast<const uintx4*>(x + chunk * 128);
    const int at = min((int)fast_div((unsigned)(chunk * 4 + step), per_group), l.groups - 1) * 16;
    sc[d] = *reinterpret_cast<const four*>(scales + at);
    zp[d] = a.zeros ? *reinterpret_cast<const unsigned*>(zeros + at) : 0x08080808u;
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (first + d < last) load(first + d, d);
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  floatx4 sum = {0, 0, 0, 0};
  for (int c0 = first; c0 < last; c0 += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int chunk = c0 + d;
      if (chunk < last) {
        const vec xb = __builtin_bit_cast(vec, xv[d]);
        const floatx4 none = {0, 0, 0, 0};
        const floatx4 xs = C::mfma(ones, xb, none);
        floatx4 p[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) p[s] = C::mfma(widen<T>(codes[d][s]), xb, none);
        const four f = sc[d];
        const unsigned z = zp[d];
        if (chunk + DEPTH < last) load(chunk + DEPTH, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = step & 1 ? p[1][i] : p[0][i], hi = step & 1 ? p[3][i] : p[2][i];
          const float v = step & 2 ? hi : lo;
          sum[i] = fmaf((float)f[i], fmaf(-16.f - (float)((z >> (8 * i)) & 255u), xs[i], v), sum[i]);
        }
      }
    }
  }
  // the four columns of a row
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum[i] += __shfl_xor(sum[i], 1, 64);
    sum[i] += __shfl_xor(sum[i], 2, 64);
  }
  if (step == 0) part[wave][row * 4 + g] = sum;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  // lane: unit lane % 16 of the tile, row lane / 16
  const int r = lane >> 4, j = lane & 15;
  float v = 0.f;
#pragma unroll
  for (int u = 0; u < W; ++u) v += part[u][r * 4 + (j >> 2)][j & 3];
  if (r < a.m && tile * 16 + j < a.n) finish<T>(a, r, tile * 16 + j, v);
}

// Few rows.  NT tiles of 16 units and RT tiles of 16 rows to a wave, W waves share the reduction out in chunks of 128; DEPTH chunks of
// codes and of x are on their way.  A lane's x belongs to row 16 rt + lane % 16: lanes of rows that are not there load nothing, so that one row costs
// the memory pipe a 16th of what 16 cost it.
template <typename T, int NT, int RT, int W, int DEPTH>
__global__ __launch_bounds__(W * 64) void w4_rows_kernel(const W4Args a, const W4Layout l) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  __shared__ floatx4 part[W][NT * RT][64];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int tile0 = (int)blockIdx.x * NT, m0 = (int)blockIdx.y * 16 * RT;
  const int g = lane >> 4, col = lane & 15;
  const unsigned char* base = static_cast<const unsigned char*>(a.packed);
  const int first = l.chunks * wave / W, last = l.chunks * (wave + 1) / W;
  const uintx4* w[NT];
  const T* scales[NT];
  const unsigned char* zeros[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tile = min(tile0 + t, l.tiles - 1);   // (a tile past the last is computed again and not stored)
    w[t] = reinterpret_cast<const uintx4*>(base) + (size_t)tile * l.chunks * 64 + lane;
    // this lane's sums belong to units 4 g .. 4 g + 3 of the tile
    scales[t] = reinterpret_cast<const T*>(base + l.scales_at) + (size_t)tile * l.groups * 16 + 4 * g;
    zeros[t] = base + l.zeros_at + (size_t)tile * l.groups * 16 + 4 * g;
  }
  const T* x[RT];
  bool row_ok[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = m0 + r * 16 + col;
    row_ok[r] = row < a.m;
    x[r] = static_cast<const T*>(a.x) + (long)min(row, a.m - 1) * a.x_stride + 8 * g;
  }
  uintx4 codes[DEPTH][NT], xv[DEPTH][4][RT];
  auto load = [&](int chunk, int d) {
#pragma unroll
    for (int t = 0; t < NT; ++t) codes[d][t] = w[t][(size_t)chunk * 64];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int k = chunk * 128 + s * 32;
        xv[d][s][r] = (uintx4){0, 0, 0, 0};
        if (row_ok[r] && k + 8 * g < a.k) xv[d][s][r] = *reinterpret_cast<const uintx4*>(x[r] + k);
      }
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (first + d < last) load(first + d, d);
  // scales and 16 + zero points of the group at hand
  const int per_group = a.group / 32;
  int gr = first * 4 / per_group, left = per_group - (first * 4 - gr * per_group);   // (steps left in it)
  typedef T four __attribute__((ext_vector_type(4)));
  four sc[NT];
  unsigned zp[NT];
  auto load_group = [&]() {
    const int at = min(gr, l.groups - 1) * 16;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      sc[t] = *reinterpret_cast<const four*>(scales[t] + at);
      zp[t] = a.zeros ? *reinterpret_cast<const unsigned*>(zeros[t] + at) : 0x08080808u;
    }
  };
  load_group();
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  floatx4 sum[NT][RT], acc[NT][RT], xs[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    xs[r] = (floatx4){0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[t][r] = acc[t][r] = (floatx4){0, 0, 0, 0};
  }
  auto flush = [&]() {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float z = -16.f - (float)((zp[t] >> (8 * i)) & 255u), f = (float)sc[t][i];
#pragma unroll
        for (int r = 0; r < RT; ++r) sum[t][r][i] = fmaf(f, fmaf(z, xs[r][i], acc[t][r][i]), sum[t][r][i]);
      }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      xs[r] = (floatx4){0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t][r] = (floatx4){0, 0, 0, 0};
    }
  };
  for (int c0 = first; c0 < last; c0 += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int chunk = c0 + d;
      if (chunk < last) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
          for (int r = 0; r < RT; ++r) xs[r] = C::mfma(ones, __builtin_bit_cast(vec, xv[d][s][r]), xs[r]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const vec wv = widen<T>(codes[d][t][s]);
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[t][r] = C::mfma(wv, __builtin_bit_cast(vec, xv[d][s][r]), acc[t][r]);
          }
          if (--left == 0) {
            flush();
            ++gr;
            left = per_group;
            load_group();
          }
        }
        if (chunk + DEPTH < last) load(chunk + DEPTH, d);
      }
    }
  }
  flush();   // (a group that goes on in the next wave's part, or that the row ends in)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) part[wave][t * RT + r][lane] = sum[t][r];
  __syncthreads();
  for (int i = (int)threadIdx.x; i < NT * RT * 64; i += W * 64) {
    const int which = i >> 6, ln = i & 63;
    floatx4 v = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < W; ++u) v += part[u][which][ln];
    const int row = m0 + (which % RT) * 16 + (ln & 15), j0 = (tile0 + which / RT) * 16 + 4 * (ln >> 4);
    if (row >= a.m) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j0 + e < a.n) finish<T>(a, row, j0 + e, v[e]);
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

namespace {
#ifndef D2
#define D2 3
#endif
#ifndef D1
#define D1 4
#endif
template <typename T>
hipError_t launch_type(const W4Args& a, const W4Layout& l, hipStream_t st) {
  auto go = [&](auto kernel, int nt, int rt) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((l.tiles + nt - 1) / nt), (unsigned)((a.m + 16 * rt - 1) / (16 * rt))), dim3(512), 0, st, a, l);
    return hipGetLastError();
  };
  if (a.m <= 4) {
    hipLaunchKernelGGL((w4_few_kernel<T, 8, D1>), dim3((unsigned)l.tiles), dim3(512), 0, st, a, l, make_fastdiv((uint32_t)a.group / 32));
    return hipGetLastError();
  }
  if (a.m <= 16) return go(w4_rows_kernel<T, 1, 1, 8, D2>, 1, 1);
  return go(w4_rows_kernel<T, 2, 2, 8, 2>, 2, 2);
}
}  // namespace

hipError_t launch_w4(const W4Args& a, int dtype, hipStream_t st) {
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.zeros != 0);
  return dtype == T_F16 ? launch_type<_Float16>(a, l, st) : launch_type<__bf16>(a, l, st);
}

}  // namespace relay
