// Norms before and after a block, with its gate and the residual stream:  s = alpha r + beta gate post(x),  y = pre(s).
//
// Bytes: x and r are read once, s and y written once, and nothing else leaves the registers of the threads that share a row.  A mean is
// formed before the squares of what lies off it (not as a difference of two sums, which loses a row whose mean is large), for which the row is at hand anyway.
// 8192 rows of 8192 bf16: 97 us, 5.5 TB/s, as fast as a large copy.  1003 rows of 5003 fp16, three reductions, a gate and four parameters: 16.3 us, one round of workgroups, each of which waits for its
// loads, its reductions and its parameters in turn (the bytes take 8; with 512 threads to a row 18.0, with 16-byte aligned pieces and two ends 17.1, with the parameters asked for ahead 18).
#include <type_traits>

#include "decoder_ops.hpp"
#include "wave_ops.hpp"

namespace relay {
namespace {

template <typename T> struct Piece { typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));

// TPR threads share a row, P pieces of 16 bytes each: piece i of a thread begins at channel (i TPR + thread) V.  Pieces are loaded at the alignment of the
// element type, so rows of odd lengths take the same path; the one that ends a row short is taken element by element.
template <typename T, int TPR, int P>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void residual_norm_kernel(const NormArgs a) {
  constexpr int V = 16 / sizeof(T), ROWS = TPR < 256 ? 256 / TPR : 1, W = TPR / 64;
  typedef typename Piece<T>::vec vec;
  __shared__ float part[2][W > 1 ? W : 1];
  const int at = (int)threadIdx.x % TPR, row = (int)blockIdx.x * ROWS + (int)threadIdx.x / TPR, c = a.channels;
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
      for (int u = 0; u < W; ++u) v += part[turn][u];
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

template <typename T, int TPR, int P>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  constexpr int kMost = 1 << 21;   // workgroups of a launch: one has fewer than 2^32 threads
  for (long first = 0; first < a.tokens; first += (long)kMost * ROWS) {
    NormArgs b = a;
    b.tokens = (int)(a.tokens - first < (long)kMost * ROWS ? a.tokens - first : (long)kMost * ROWS);
    auto on = [&](auto*& p, int64_t stride) {
      if (p) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)(first * stride * (int64_t)sizeof(T)));
    };
    on(b.x, a.x_stride), on(b.res, a.res_stride), on(b.gate, a.gate_stride), on(b.sum, a.sum_stride), on(b.y, a.y_stride);
    hipLaunchKernelGGL((residual_norm_kernel<T, TPR, P>), dim3((unsigned)((b.tokens + ROWS - 1) / ROWS)), dim3(TPR * ROWS), 0, st, b);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_type(const NormArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int pieces = (a.channels + V - 1) / V;
  // (A wave to a row needs no barrier.  Few rows: twice the threads, half the chain; many: workgroups of 256, of which more fit a CU.  The 1003 rows above 16.3 us with 256 and four pieces, 18.0 with 512 and two.)
  if (pieces <= 64) return launch<T, 64, 1>(a, st);
  if (pieces <= 128) return launch<T, 64, 2>(a, st);
  if (pieces <= 256) return launch<T, 256, 1>(a, st);
  if (pieces <= 512) return a.tokens < 512 ? launch<T, 512, 1>(a, st) : launch<T, 256, 2>(a, st);
  if (pieces <= 1024) return a.tokens < 512 ? launch<T, 512, 2>(a, st) : launch<T, 256, 4>(a, st);
  if (pieces <= 2048) return launch<T, 512, 4>(a, st);
  return launch<T, 1024, 4>(a, st);
}

}  // namespace

hipError_t launch_residual_norm(const NormArgs& a, int dtype, hipStream_t st) {
  if (dtype == T_F16) return launch_type<_Float16>(a, st);
  return dtype == T_BF16 ? launch_type<__bf16>(a, st) : launch_type<float>(a, st);
}

}  // namespace relay
