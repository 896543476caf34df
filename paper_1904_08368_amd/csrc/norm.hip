// Norms before and after a block, with its gate and the residual stream:  s = alpha r + beta gate post(x),  y = pre(s).
//
// Bytes: x and r are read once, s and y written once, and nothing else leaves the registers of the threads that share a row.  A mean is
// formed before the squares of what lies off it (not as a difference of two sums, which loses a row whose mean is large), for which the row is at hand anyway.
// 8192 rows of 8192 bf16: 97 us, 5.5 TB/s, as fast as a large copy.  1003 rows of 5003 fp16, three reductions, a gate and four parameters: 15 us, one round of workgroups, each of which waits for its
// loads, its reductions and its parameters in turn (the bytes take 8; with pieces that are 16-byte aligned and two ends 5 % more, with the parameters asked for ahead 10 %).
#include <type_traits>

#include "decoder_ops.hpp"
#include "wave_ops.hpp"

namespace relay {
namespace {

template <typename T> struct Piece { typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));

// TPR threads share a row, P pieces of 16 bytes each: piece i of a thread begins at channel (i TPR + thread) V.  Pieces are loaded at the alignment of the
// element type, so rows of odd lengths take the same path; the one that ends a row short is taken element by element.
// MOST 64: TPR is 64, four rows to a workgroup; more: a row to a workgroup of up to as many.
template <typename T, int MOST, int P>
__global__ __launch_bounds__((MOST < 256 ? 256 : MOST)) void residual_norm_kernel(const NormArgs a) {
  constexpr int V = 16 / sizeof(T), ROWS = MOST < 256 ? 256 / MOST : 1, W = MOST / 64;
  typedef typename Piece<T>::vec vec;
  __shared__ float part[2][W];
  const int TPR = W == 1 ? 64 : (int)blockDim.x, waves = TPR / 64, at = W == 1 ? (int)threadIdx.x % 64 : (int)threadIdx.x;
  const int row = (int)blockIdx.x * ROWS + (W == 1 ? (int)threadIdx.x / 64 : 0), c = a.channels;
  if (ROWS > 1 && row >= a.tokens) return;   // (whole waves: nothing below waits for them)
  auto load = [&](const void* p, int64_t stride, vec (&v)[P]) {
    const T* const src = static_cast<const T*>(p) + row * stride;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int j = (i * TPR + at) * V;
      if (j + V <= c) {
        v[i] = *reinterpret_cast<const vec*>(src + j);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] = j + e < c ? src[j + e] : (T)0.f;
      }
    }
  };
  auto store = [&](void* p, int64_t stride, const float (&v)[P][V]) {
    T* const dst = static_cast<T*>(p) + row * stride;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int j = (i * TPR + at) * V;
      vec o;
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (T)v[i][e];
      if (j + V <= c) {
        *reinterpret_cast<vec*>(dst + j) = o;
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (j + e < c) dst[j + e] = o[e];
      }
    }
  };
  int turn = 0;
  auto row_sum = [&](float v) {   // over the threads of the row
    v = wave_sum(v);
    if constexpr (W > 1) {
      if ((at & 63) == 0) part[turn][at >> 6] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int u = 0; u < W; ++u) v += u < waves ? part[turn][u] : 0.f;
      turn ^= 1;   // (the other half: whoever is late still reads this one)
    }
    return v;
  };
  float b[P][V];
  auto norm = [&](int kind, float eps, const float* weight, const float* bias) {
    if (kind == N_LAYER) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) m += b[i][e];
      m = row_sum(m) / (float)c;   // (divided: a row that is all alike then has its own value as mean, and nothing off it)
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) b[i][e] = (i * TPR + at) * V + e < c ? b[i][e] - m : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) q = fmaf(b[i][e], b[i][e], q);
    const float k = 1.f / sqrtf(row_sum(q) / (float)c + eps);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int j = (i * TPR + at) * V;
      if (j + V <= c) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          floatx4u w = {1.f, 1.f, 1.f, 1.f}, z = {0.f, 0.f, 0.f, 0.f};
          if (weight) w = *reinterpret_cast<const floatx4u*>(weight + j + e);
          if (bias) z = *reinterpret_cast<const floatx4u*>(bias + j + e);
#pragma unroll
          for (int f = 0; f < 4; ++f) b[i][e + f] = fmaf(b[i][e + f] * k, w[f], z[f]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (j + e < c) b[i][e] = fmaf(b[i][e] * k, weight ? weight[j + e] : 1.f, bias ? bias[j + e] : 0.f);
      }
    }
  };
  vec xv[P], rv[P], gv[P];
  load(a.x, a.x_stride, xv);
  if (a.res) load(a.res, a.res_stride, rv);
  if (a.gate) load(a.gate, a.gate_stride, gv);
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) b[i][e] = (float)xv[i][e];
  if (a.post != N_NONE) norm(a.post, a.post_eps, a.post_weight, a.post_bias);
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (a.gate) b[i][e] *= (float)gv[i][e];
      b[i][e] *= a.branch_scale;
      if (a.res) b[i][e] = fmaf((float)rv[i][e], a.residual_scale, b[i][e]);
    }
  if (a.sum) store(a.sum, a.sum_stride, b);
  if (a.pre != N_NONE) {
    norm(a.pre, a.pre_eps, a.pre_weight, a.pre_bias);
    store(a.y, a.y_stride, b);
  }
}

template <typename T, int MOST, int P>
hipError_t launch(const NormArgs& a, int pieces, hipStream_t st) {
  constexpr int ROWS = MOST < 256 ? 256 / MOST : 1;
  constexpr int kMost = 1 << 21;   // workgroups of a launch: one has fewer than 2^32 threads
  const int threads = MOST < 256 ? 256 : (pieces + 64 * P - 1) / (64 * P) * 64;   // (no wave without a piece)
  for (long first = 0; first < a.tokens; first += (long)kMost * ROWS) {
    NormArgs b = a;
    b.tokens = (int)(a.tokens - first < (long)kMost * ROWS ? a.tokens - first : (long)kMost * ROWS);
    auto on = [&](auto*& p, int64_t stride) {
      if (p) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)(first * stride * (int64_t)sizeof(T)));
    };
    on(b.x, a.x_stride), on(b.res, a.res_stride), on(b.gate, a.gate_stride), on(b.sum, a.sum_stride), on(b.y, a.y_stride);
    hipLaunchKernelGGL((residual_norm_kernel<T, MOST, P>), dim3((unsigned)((b.tokens + ROWS - 1) / ROWS)), dim3(threads), 0, st, b);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_type(const NormArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int pieces = (a.channels + V - 1) / V;
  // A wave to a row needs no barrier.  More pieces: as few to a thread as leave a CU four workgroups, and no more waves than have some.  us, fp16, 1000 rows (4000 with two norms, gate and biases):
  // 2560 channels on 256 threads / the 192 that have pieces 6.9 (23.2) / 6.4 (21.9); 7168 four pieces to a thread / two 12.8 (66.9) / 11.3 (69.1), 8192 13.0 (70.5) / 12.1 (78.6); 12000 four / three
  // 23.2 (125) / 20.8 (114).
  if (pieces <= 64) return launch<T, 64, 1>(a, pieces, st);
  if (pieces <= 128) return launch<T, 64, 2>(a, pieces, st);
  if (pieces <= 256 || (pieces <= 512 && a.tokens < 512)) return launch<T, 512, 1>(a, pieces, st);
  if (pieces <= 896 || (pieces <= 1024 && a.tokens < 512)) return launch<T, 512, 2>(a, pieces, st);
  if (pieces > 1024 && pieces <= 1536) return launch<T, 512, 3>(a, pieces, st);
  if (pieces <= 2048) return launch<T, 512, 4>(a, pieces, st);
  return launch<T, 1024, 4>(a, pieces, st);
}

}  // namespace

hipError_t launch_residual_norm(const NormArgs& a, int dtype, hipStream_t st) {
  if (dtype == T_F16) return launch_type<_Float16>(a, st);
  return dtype == T_BF16 ? launch_type<__bf16>(a, st) : launch_type<float>(a, st);
}

}  // namespace relay
