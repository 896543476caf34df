// The router of a mixture of experts:  l = W x,  score = softmax(l) or sigmoid(l),  the top_k of score + bias and their weights.
//
// Two experts next to each other must not change places with the order of a sum, so products are added up in 64 bits (a product of two 16-bit
// numbers is exact there).  The workgroup that is last to leave its part of the logits of a tile of tokens makes the choice for them: one launch.
// One token, 64 experts by 4096 channels, bf16: 6.2 us, loads, one exchange between workgroups and eight choices in turn.  509 tokens, 128 experts, fp16: 19.9 us, of which the products on the matrix
// cores of 64 bits, 43 % of the clocks, would be 8 (with products by vector instructions the call took 130); a last workgroup chooses for its 16 tokens in 4.
#include "decoder_ops.hpp"
#include "wave_ops.hpp"

namespace relay {
namespace {

typedef unsigned long long u64;
typedef double doublex4 __attribute__((ext_vector_type(4)));

// ascending with the value; a NaN is less than everything else, and 0 is what has been taken
__device__ __forceinline__ u64 key_of(double v) {
  if (!(v == v)) return 1;
  const long long b = __builtin_bit_cast(long long, v + 0.0);
  return (u64)b ^ ((u64)(b >> 63) | 0x8000000000000000ull);
}

__device__ __forceinline__ unsigned wave_max32(unsigned v) {
  return wave_fold32(v, [](unsigned a, unsigned b) { return a > b ? a : b; });
}

// The choice for token t, by one wave.  Lane l holds experts l, l + 64, ..: score comes as their logits.
template <int PER>
__device__ __forceinline__ void choose(const RouteArgs& a, double (&score)[PER], int t, int lane) {
  if (a.score == S_SOFTMAX) {
    double top = -__builtin_inf();
#pragma unroll
    for (int i = 0; i < PER; ++i) top = score[i] > top ? score[i] : top;
    top = wave_fold64(top, [](double x, double y) { return x > y ? x : y; });
    double all = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      score[i] = i * 64 + lane < a.experts ? exp(score[i] - top) : 0.0;
      all += score[i];
    }
    all = 1.0 / wave_sum64(all);
#pragma unroll
    for (int i = 0; i < PER; ++i) score[i] *= all;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) score[i] = 1.0 / (1.0 + exp(-score[i]));
  }
  unsigned hi[PER], lo[PER];   // the halves of a score's key: most choices are made by the upper ones
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * 64 + lane;
    const u64 key = e < a.experts ? key_of(a.bias ? score[i] + (double)a.bias[e] : score[i]) : 0;
    hi[i] = (unsigned)(key >> 32);
    lo[i] = (unsigned)key;
  }
  int mine = 0;
  double weight = 0, sum = 0;   // of slot `lane`; of all slots
  for (int s = 0; s < a.top_k; ++s) {
    unsigned best = hi[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = hi[i] > best ? hi[i] : best;
    best = __builtin_amdgcn_readfirstlane(wave_max32(best));
    int many = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) many += __builtin_popcountll(__ballot(hi[i] == best));
    unsigned low = 0;
    if (many > 1) {
#pragma unroll
      for (int i = 0; i < PER; ++i) low = hi[i] == best && lo[i] > low ? lo[i] : low;
      low = __builtin_amdgcn_readfirstlane(wave_max32(low));
    }
    // the first that has it
    int at = 0;
    double w = 0;
    bool taken = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const u64 has = __ballot(hi[i] == best && (many == 1 || lo[i] == low));
      if (has && !taken) {
        const int l = __builtin_ctzll(has);
        const u64 bits = __builtin_bit_cast(u64, score[i]);
        at = i * 64 + l;
        w = __builtin_bit_cast(double, (u64)(unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)bits, l));
        if (lane == l) hi[i] = lo[i] = 0;
        taken = true;
      }
    }
    sum += w;
    if (lane == s) mine = at, weight = w;
  }
  if (lane >= a.top_k) return;
  if (a.normalize) weight = sum == 0 ? 0.0 : weight / sum;
  a.chosen[(size_t)t * a.top_k + lane] = mine;
  a.weights[(size_t)t * a.top_k + lane] = (float)(weight * (double)a.scale);
}

// Logit e of token t: the sum of its parts.
__device__ __forceinline__ double logit_of(const RouteArgs& a, int t, int e) {
  double v = 0, part[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    part[i] = __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const u64*>(a.logits) + ((size_t)min(i, a.splits - 1) * a.tokens + t) * a.experts + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
#pragma unroll
  for (int i = 0; i < 4; ++i) v += i < a.splits ? part[i] : 0.0;
  return v;
}

// Behind the stores of a workgroup's logits: whoever is the last of `arrivals` for a tile of tokens chooses for all of them.
// held: LDS for the logits of W tokens by up to kHeld experts, which all threads fetch together.
constexpr int kHeld = 256;
template <int W, bool HELD>
__device__ __forceinline__ void choose_last(const RouteArgs& a, int tile, int arrivals, int t0, int rows, bool* last, double* held) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned* const cell = a.counters + (size_t)tile * 16;
    const unsigned old = __hip_atomic_fetch_add(cell, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = old == (unsigned)arrivals - 1;
    if (*last) __hip_atomic_store(cell, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!*last) return;
  if constexpr (HELD) {
    for (int r0 = 0; r0 < rows; r0 += W) {
      const int many = min(W, rows - r0) * a.experts;   // (rows of tokens one behind the other)
      for (int i = (int)threadIdx.x; i < many; i += W * 64) held[i] = logit_of(a, t0 + r0 + i / a.experts, i % a.experts);
      __syncthreads();
      auto pick = [&](auto& score, int per) {
#pragma unroll
        for (int i = 0; i < per; ++i) score[i] = i * 64 + lane < a.experts ? held[wave * a.experts + i * 64 + lane] : -__builtin_inf();
        choose(a, score, t0 + r0 + wave, lane);
      };
      if (r0 + wave < rows) {
        double one[1], two[2], four[4];
        if (a.experts <= 64) pick(one, 1);
        else if (a.experts <= 128) pick(two, 2);
        else pick(four, 4);
      }
      __syncthreads();
    }
  } else for (int r = wave; r < rows; r += W) {
    double score[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) score[i] = i * 64 + lane < a.experts ? logit_of(a, t0 + r, i * 64 + lane) : -__builtin_inf();
    choose(a, score, t0 + r, lane);
  }
}
__device__ __forceinline__ void leave(const RouteArgs& a, int z, int t, int e, double v) {
  __hip_atomic_store(reinterpret_cast<u64*>(a.logits) + ((size_t)z * a.tokens + t) * a.experts + e, __builtin_bit_cast(u64, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Few tokens: a workgroup to an expert, its threads share the channels out.
constexpr int kFewTokens = 4;
template <typename T>
__global__ __launch_bounds__(256) void route_few_kernel(const RouteArgs a) {
  typedef T vec __attribute__((ext_vector_type(8)));
  __shared__ double part[4][kFewTokens], held[4 * kHeld];
  __shared__ bool last;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, e = (int)blockIdx.x;
  const T* const w = static_cast<const T*>(a.w) + (size_t)e * a.channels;
  const T* const x = static_cast<const T*>(a.x);
  double sum[kFewTokens];
#pragma unroll
  for (int r = 0; r < kFewTokens; ++r) sum[r] = 0;
  for (int c = tid * 8; c < a.channels; c += 2048) {
    const vec wv = *reinterpret_cast<const vec*>(w + c);
#pragma unroll
    for (int r = 0; r < kFewTokens; ++r)
      if (r < a.tokens) {
        const vec xv = *reinterpret_cast<const vec*>(x + (size_t)r * a.x_stride + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[r] = fma((double)(float)wv[i], (double)(float)xv[i], sum[r]);   // (in 32 bits a product of two bf16 numbers may leave the range)
      }
  }
#pragma unroll
  for (int r = 0; r < kFewTokens; ++r)
    if (r < a.tokens) {
      const double v = wave_sum64(sum[r]);
      if (lane == 0) part[wave][r] = v;
    }
  __syncthreads();
  if (tid < a.tokens) leave(a, 0, tid, e, part[0][tid] + part[1][tid] + (part[2][tid] + part[3][tid]));
  if (a.experts <= kHeld) choose_last<4, true>(a, 0, a.experts, 0, a.tokens, &last, held);
  else choose_last<4, false>(a, 0, a.experts, 0, a.tokens, &last, held);
}

// More: a workgroup makes 16 tokens by 16 experts on the matrix cores of 64 bits, its waves and, where there are few such tiles, several workgroups
// share the channels out.  A lane loads eight channels of a row at once; which of them meet in which instruction does not matter as long as x and w agree.
// W waves: 16, one to each choice, where there are more than eight and lanes hold few experts (us, 8 / 16 waves, 64 experts by 4096 channels: 8 tokens 9.4 / 11.6, 16 13.1 / 12.9; 128
// experts: 16 tokens 15.7 / 15.1, 509 23.4 / 20.7).
constexpr int kTileTokens = 16;
template <typename T, int W, bool HELD>
__global__ __launch_bounds__(W * 64) void route_tiles_kernel(const RouteArgs a) {
  typedef T vec __attribute__((ext_vector_type(8)));
  static_assert(kHeld <= 256, "the waves' sums make room for the logits");
  __shared__ double part[W][256];
  __shared__ bool last;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
  const int e0 = (int)blockIdx.x * 16, t0 = (int)blockIdx.y * 16, z = (int)blockIdx.z;
  const int blocks = (a.channels + 31) / 32, shares = W * a.splits, share = z * W + wave;
  // (rows that are not there repeat the last one, and are not stored)
  const T* const x = static_cast<const T*>(a.x) + (size_t)min(t0 + col, a.tokens - 1) * a.x_stride + g * 8;
  const T* const w = static_cast<const T*>(a.w) + (size_t)min(e0 + col, a.experts - 1) * a.channels + g * 8;
  constexpr int D = 4;
  vec xv[D], wv[D];
  auto load = [&](int i, int block) {
    const bool there = block < blocks && block * 32 + g * 8 < a.channels;
    xv[i] = wv[i] = (vec){};
    if (there) {
      xv[i] = *reinterpret_cast<const vec*>(x + block * 32);
      wv[i] = *reinterpret_cast<const vec*>(w + block * 32);
    }
  };
  doublex4 sum = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < D; ++i) load(i, share + i * shares);
  for (int block = share; block < blocks; block += D * shares) {   // (the waves of a workgroup side by side along the rows)
#pragma unroll
    for (int i = 0; i < D; ++i) {
#pragma unroll
      for (int c = 0; c < 8; ++c) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)wv[i][c], (double)(float)xv[i][c], sum, 0, 0, 0);
      load(i, block + (D + i) * shares);
    }
  }
  // a lane holds token `col` and experts g, g + 4, g + 8, g + 12 of the tile
#pragma unroll
  for (int i = 0; i < 4; ++i) part[wave][(4 * i + g) * 16 + col] = sum[i];
  __syncthreads();
  if (tid < 256) {
    double v = 0;
#pragma unroll
    for (int u = 0; u < W; ++u) v += part[u][tid];
    const int e = e0 + (tid >> 4), t = t0 + (tid & 15);
    if (e < a.experts && t < a.tokens) leave(a, z, t, e, v);
  }
  choose_last<W, HELD>(a, (int)blockIdx.y, (int)(gridDim.x * gridDim.z), t0, min(kTileTokens, a.tokens - t0), &last, part[0]);
}

// Arrival counters lie 64 bytes apart in front of the workspace, in a region that is the same for every call; behind them the logits of as many tokens as a launch takes.
constexpr int kRouteTiles = 256;
constexpr size_t kRouteCounterBytes = (size_t)kRouteTiles * 64;
constexpr int kAtOnce = kRouteTiles * kTileTokens;

// workgroups that share a tile's channels: as many as leave every CU one
int splits_of(int tokens, int experts, int channels) {
  if (tokens <= kFewTokens) return 1;
  const int tiles = (tokens + 15) / 16 * ((experts + 15) / 16), most = channels / 512;   // (a block of 32 to a wave at least)
  int s = 256 / tiles;
  s = s < most ? s : most;
  return s < 1 ? 1 : s > 4 ? 4 : s;   // (four: what the last workgroup fetches of a logit at once)
}

size_t route_bytes(const RouteArgs& a, int parts) { return kRouteCounterBytes + ((size_t)parts * a.experts * 8 + 255) / 256 * 256; }

}  // namespace

size_t route_workspace_need(const RouteArgs& a) {
  const int tokens = a.tokens < kAtOnce ? a.tokens : kAtOnce;
  return route_bytes(a, tokens * splits_of(tokens, a.experts, a.channels));
}
size_t route_workspace_bytes(const RouteArgs& a) {
  const int tokens = a.tokens < kAtOnce ? a.tokens : kAtOnce;
  int most = tokens;   // parts of an expert's logits: tokens times splits
  for (int s = 2; s <= 4; ++s) {
    const int up_to = 16 * (256 / s / ((a.experts + 15) / 16)), t = tokens < up_to ? tokens : up_to;   // the most tokens that may have as many splits
    if (t > 0 && splits_of(t, a.experts, a.channels) >= s && t * s > most) most = t * s;
  }
  return route_bytes(a, most);
}

hipError_t launch_route(const RouteArgs& args, int dtype, hipStream_t st) {
  for (long first = 0; first < args.tokens; first += kAtOnce) {
    RouteArgs a = args;
    a.tokens = (int)(args.tokens - first < kAtOnce ? args.tokens - first : kAtOnce);
    a.x = static_cast<const char*>(args.x) + first * args.x_stride * 2;
    a.chosen = args.chosen + first * args.top_k;
    a.weights = args.weights + first * args.top_k;
    a.counters = static_cast<unsigned*>(args.workspace);
    a.logits = reinterpret_cast<double*>(static_cast<char*>(args.workspace) + kRouteCounterBytes);
    a.splits = splits_of(a.tokens, a.experts, a.channels);
    if (a.tokens <= kFewTokens) {
      const dim3 grid((unsigned)a.experts), block(256);
      if (dtype == T_F16) hipLaunchKernelGGL((route_few_kernel<_Float16>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((route_few_kernel<__bf16>), grid, block, 0, st, a);
    } else {
      const dim3 grid((unsigned)((a.experts + 15) / 16), (unsigned)((a.tokens + 15) / 16), (unsigned)a.splits);
      const bool held = a.experts <= kHeld;
      if (held && a.tokens > 8) {
        if (dtype == T_F16) hipLaunchKernelGGL((route_tiles_kernel<_Float16, 16, true>), grid, dim3(1024), 0, st, a);
        else hipLaunchKernelGGL((route_tiles_kernel<__bf16, 16, true>), grid, dim3(1024), 0, st, a);
      } else if (held) {
        if (dtype == T_F16) hipLaunchKernelGGL((route_tiles_kernel<_Float16, 8, true>), grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((route_tiles_kernel<__bf16, 8, true>), grid, dim3(512), 0, st, a);
      } else if (dtype == T_F16) {
        hipLaunchKernelGGL((route_tiles_kernel<_Float16, 8, false>), grid, dim3(512), 0, st, a);
      } else {
        hipLaunchKernelGGL((route_tiles_kernel<__bf16, 8, false>), grid, dim3(512), 0, st, a);
      }
    }
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace relay
