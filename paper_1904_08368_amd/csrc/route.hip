// The router of a mixture of experts:  l = W x,  score = softmax(l) or sigmoid(l),  the top_k of score + bias and their weights.
//
// Two experts next to each other must not change places with the order of a sum, so products are added up in 64 bits (a product of two 16-bit
// numbers is exact in 32).  The workgroup that is last to leave its experts' logits of a tile of tokens makes the choice for them: one launch.
#include "decoder_ops.hpp"
#include "wave_ops.hpp"

namespace relay {
namespace {

typedef unsigned long long u64;
constexpr int kRouteTokens = 16;   // a tile

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// ascending with the value; a NaN is less than everything else, and 0 is what has been taken
__device__ __forceinline__ u64 key_of(double v) {
  if (!(v == v)) return 1;
  const long long b = __builtin_bit_cast(long long, v + 0.0);
  return (u64)b ^ ((u64)(b >> 63) | 0x8000000000000000ull);
}

// The choice for token t, by one wave.  Lane l holds experts l, l + 64, ..
template <int PER>
__device__ void choose(const RouteArgs& a, const double* logits, int t, int lane) {
  double score[PER];
  u64 by[PER];
  double most = -__builtin_inf();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * 64 + lane;
    score[i] = e < a.experts ? __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const u64*>(logits) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) : -__builtin_inf();
    most = score[i] > most ? score[i] : most;
  }
  if (a.score == S_SOFTMAX) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double o = __shfl_xor(most, d);
      most = o > most ? o : most;
    }
    double all = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      score[i] = i * 64 + lane < a.experts ? exp(score[i] - most) : 0.0;
      all += score[i];
    }
    all = wave_sum64(all);
#pragma unroll
    for (int i = 0; i < PER; ++i) score[i] /= all;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) score[i] = 1.0 / (1.0 + exp(-score[i]));
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * 64 + lane;
    by[i] = e < a.experts ? key_of(a.bias ? score[i] + (double)a.bias[e] : score[i]) : 0;
  }
  int mine = 0;
  double weight = 0, sum = 0;   // of slot `lane`; of all slots
  for (int s = 0; s < a.top_k; ++s) {
    u64 best = 0;
    int at = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (by[i] > best) best = by[i], at = i * 64 + lane;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 o = __shfl_xor(best, d);
      const int oi = __shfl_xor(at, d);
      if (o > best || (o == best && oi < at)) best = o, at = oi;
    }
    double w = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i * 64 + lane == at) {
        by[i] = 0;
        w = score[i];
      }
    w = __shfl(w, at & 63);
    sum += w;
    if (lane == s) mine = at, weight = w;
  }
  if (lane >= a.top_k) return;
  if (a.normalize) weight = sum == 0 ? 0.0 : weight / sum;
  a.chosen[(size_t)t * a.top_k + lane] = mine;
  a.weights[(size_t)t * a.top_k + lane] = (float)(weight * (double)a.scale);
}

// A workgroup: one expert, a tile of tokens.  Its threads share the channels out.
template <typename T>
__global__ __launch_bounds__(256) void route_kernel(const RouteArgs a) {
  typedef T vec __attribute__((ext_vector_type(8)));
  __shared__ double part[4][kRouteTokens];
  __shared__ bool s_last;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, e = (int)blockIdx.x, t0 = (int)blockIdx.y * kRouteTokens;
  const int rows = min(kRouteTokens, a.tokens - t0);
  const T* const w = static_cast<const T*>(a.w) + (size_t)e * a.channels;
  const T* const x = static_cast<const T*>(a.x) + (size_t)t0 * a.x_stride;
  double sum[kRouteTokens];
#pragma unroll
  for (int r = 0; r < kRouteTokens; ++r) sum[r] = 0;
  for (int c = tid * 8; c < a.channels; c += 2048) {
    const vec wv = *reinterpret_cast<const vec*>(w + c);
#pragma unroll
    for (int r = 0; r < kRouteTokens; ++r)
      if (r < rows) {
        const vec xv = *reinterpret_cast<const vec*>(x + (size_t)r * a.x_stride + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[r] += (double)((float)wv[i] * (float)xv[i]);
      }
  }
#pragma unroll
  for (int r = 0; r < kRouteTokens; ++r)
    if (r < rows) {
      const double v = wave_sum64(sum[r]);
      if (lane == 0) part[wave][r] = v;
    }
  __syncthreads();
  double* const logits = a.logits + (size_t)t0 * a.experts;
  if (tid < rows)
    __hip_atomic_store(reinterpret_cast<u64*>(logits) + (size_t)tid * a.experts + e, __builtin_bit_cast(u64, part[0][tid] + part[1][tid] + (part[2][tid] + part[3][tid])),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (wave == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the stores are this wave's)
    if (lane == 0) {
      unsigned* const cell = a.counters + (size_t)blockIdx.y * 16;
      const unsigned old = __hip_atomic_fetch_add(cell, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = old == (unsigned)a.experts - 1;
      if (s_last) __hip_atomic_store(cell, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();
  if (!s_last) return;
  for (int r = wave; r < rows; r += 4) {
    const double* const l = logits + (size_t)r * a.experts;
    if (a.experts <= 64) choose<1>(a, l, t0 + r, lane);
    else if (a.experts <= 256) choose<4>(a, l, t0 + r, lane);
    else choose<16>(a, l, t0 + r, lane);
  }
}

}  // namespace

// Arrival counters lie 64 bytes apart in front of the workspace, in a region that is the same for every call; behind them the logits of as many tokens as a launch takes.
constexpr int kRouteTiles = 256;
constexpr size_t kRouteCounterBytes = (size_t)kRouteTiles * 64;

size_t route_workspace_bytes(const RouteArgs& a) {
  const size_t tokens = a.tokens < kRouteTiles * kRouteTokens ? a.tokens : kRouteTiles * kRouteTokens;
  return kRouteCounterBytes + (tokens * a.experts * 8 + 255) / 256 * 256;
}

hipError_t launch_route(const RouteArgs& args, int dtype, hipStream_t st) {
  constexpr int most = kRouteTiles * kRouteTokens;
  for (int first = 0; first < args.tokens;) {
    RouteArgs a = args;
    const int tokens = args.tokens - first < most ? args.tokens - first : most;
    a.tokens = tokens;
    a.x = static_cast<const char*>(args.x) + (size_t)first * args.x_stride * 2;
    a.chosen = args.chosen + (size_t)first * args.top_k;
    a.weights = args.weights + (size_t)first * args.top_k;
    a.counters = static_cast<unsigned*>(args.workspace);
    a.logits = reinterpret_cast<double*>(static_cast<char*>(args.workspace) + kRouteCounterBytes);
    const dim3 grid((unsigned)a.experts, (unsigned)((tokens + kRouteTokens - 1) / kRouteTokens)), block(256);
    if (dtype == T_F16) hipLaunchKernelGGL((route_kernel<_Float16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((route_kernel<__bf16>), grid, block, 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    first += tokens;
  }
  return hipSuccess;
}

}  // namespace relay
