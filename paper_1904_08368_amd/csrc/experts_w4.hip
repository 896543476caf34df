// The experts of a mixture with 4-bit weights for a few tokens:  h = weight act(gate x) (up x),  y = sum over a token's experts of down h.
//
// A pair is a token and one of the experts it has chosen; pairs of one expert share its codes, which are most of what there is to read.  The first
// launch makes h of every pair, a workgroup to 16 units of an expert's gates and the 16 beside them; the second makes 16 channels of y, walking the units of
// all experts that were chosen, keeps a pair's part of them in LDS and adds a token's parts up in the order of its choices.  The experts' weights go into h: the second product then needs none.
// Codes become operands as in the dense kernels (16 + code, the sums of x taking the zero points out).
#include "decoder_ops.hpp"
#include "w4_common.hpp"

namespace relay {
namespace {

// The pairs that name expert e, of those from `from` on the first `most`, into rows; returns how many there are in all.  W waves, each a stretch of the pairs; two barriers.
template <int W>
__device__ int pairs_of(const int32_t* chosen, int pairs, int e, int from, int most, int* rows, int* counts) {
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int stretch = ((pairs + W - 1) / W + 63) / 64 * 64, lo = wave * stretch, hi = min(lo + stretch, pairs);
  int n = 0;
  for (int p = lo; p < hi; p += 64) n += __builtin_popcountll(__ballot(p + lane < hi && chosen[min(p + lane, hi - 1)] == e));
  if (lane == 0) counts[wave] = n;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int u = 0; u < W; ++u) {
    const int c = counts[u];
    if (u < wave) before += c;
    all += c;
  }
  if (n)
    for (int p = lo; p < hi; p += 64) {
      const bool mine = p + lane < hi && chosen[min(p + lane, hi - 1)] == e;
      const unsigned long long set = __ballot(mine);
      const int at = before + __builtin_popcountll(set & ((1ull << lane) - 1)) - from;
      if (mine && at >= 0 && at < most) rows[at] = p + lane;
      before += __builtin_popcountll(set);
    }
  __syncthreads();
  return all;
}

// What a wave holds of a chunk of 128 of the reduction: codes of NT tiles of 16 units, their scales and zero points, XL loads of four rows of x each.
// FL: steps of 32 between two applications of the scales, 4 where groups are whole chunks, 2 or 1 where they are not.
template <typename T, int NT, int XL, int FL>
struct Chunk {
  typedef T four __attribute__((ext_vector_type(4)));
  uintx4 codes[NT], x[XL];
  four scale[4 / FL][NT];
  unsigned zero[4 / FL][NT];
  // (the caller has checked that the chunk is there; rows that are not: a NULL)
  __device__ __forceinline__ void load(const unsigned char* packed, const W4Layout& l, const FastDiv& per_group, bool zeros, const long (&tile)[NT], const T* const (&row)[XL], int chunk, int k,
                                       int lane) {
    const int g = lane >> 4, col = lane & 15;
#pragma unroll
    for (int t = 0; t < NT; ++t) codes[t] = reinterpret_cast<const uintx4*>(packed)[((size_t)tile[t] * l.chunks + chunk) * 64 + lane];
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
      const int at = min((int)fast_div((unsigned)(chunk * 4 + f * FL), per_group), l.groups - 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const size_t unit = ((size_t)tile[t] * l.groups + at) * 16 + 4 * g;
        scale[f][t] = *reinterpret_cast<const four*>(packed + l.scales_at + unit * 2);
        zero[f][t] = zeros ? *reinterpret_cast<const unsigned*>(packed + l.zeros_at + unit) : 0x18181818u;
      }
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      x[i] = (uintx4){0, 0, 0, 0};
      if (row[i] && chunk * 128 + col * 8 < k) x[i] = *reinterpret_cast<const uintx4*>(row[i] + chunk * 128 + col * 8);
    }
  }
  // sums += the chunk's part; mine: LDS of this wave for XL times four rows of 16 pieces
  template <int RT>
  __device__ __forceinline__ void add(floatx4 (&sum)[NT][RT], uintx4* mine, const Widen<T>& widen, int lane) const {
    typedef W4Type<T> C;
    typedef typename C::vec vec;
    const int g = lane >> 4, col = lane & 15;
    const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
    const floatx4 none = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < XL; ++i) mine[(4 * i + g) * 16 + (col ^ ((4 * i + g) & 15))] = x[i];
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
      floatx4 acc[NT][RT], xs[RT];
#pragma unroll
      for (int s = f * FL; s < (f + 1) * FL; ++s) {
        const bool fresh = s == f * FL;
        vec xb[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const int at = XL == 1 ? col & 3 : r * 16 + col;   // (four rows: the columns behind repeat them)
          xb[r] = __builtin_bit_cast(vec, mine[at * 16 + ((4 * s + g) ^ (at & 15))]);
          xs[r] = C::mfma(ones, xb[r], fresh ? none : xs[r]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const vec wv = widen(codes[t][s]);
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[t][r] = C::mfma(wv, xb[r], fresh ? none : acc[t][r]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float z = -(float)((zero[f][t] >> (8 * i)) & 255u), k = (float)scale[f][t][i];
#pragma unroll
          for (int r = 0; r < RT; ++r) sum[t][r][i] = fmaf(k, fmaf(z, xs[r][i], acc[t][r][i]), sum[t][r][i]);
        }
    }
  }
};

__device__ __forceinline__ float activated(int act, float v) {
  return act == A_SILU ? v / (1.f + expf(-v)) : 0.5f * v * erfcf(v * -0.70710678118654752440f);   // (1 + erf(v) is erfc(-v), without the difference)
}

// A workgroup: TILES tiles of 16 units of an expert's products, its waves share the reduction out; blocks of up to XL * 4 of the expert's pairs.
//   UP: h of the pairs, from as many tiles of gates as of the other units.   not UP: a pair's part of y, in fp32.
template <typename T, bool UP, int TILES, int XL, int W, int FL>
__global__ __launch_bounds__(W * 64, 2) void experts_rows_kernel(const ExpertsArgs a, const W4Layout l, const FastDiv per_group) {
  constexpr int NT = UP ? 2 * TILES : TILES, RT = XL == 1 ? 1 : XL / 4, ROWS = XL * 4, XPIECES = ROWS * 16, SUMS = NT * RT * 64;
  __shared__ __attribute__((aligned(16))) uintx4 lds[W][XPIECES > SUMS ? XPIECES : SUMS];
  __shared__ int rows[ROWS], counts[W];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4;
  int e = (int)blockIdx.y;
  if (a.by_pair) {   // the first pair of an expert stands for it
    const int p = e;
    e = a.chosen[p];
    bool first = true;
    for (int q = lane; q < p; q += 64) first &= a.chosen[q] != e;
    if (!__all(first) || (unsigned)e >= (unsigned)a.experts) return;
  }
  const int k = UP ? a.channels : a.inter, units = (UP ? a.inter : a.channels) / 16;
  const unsigned char* const packed = static_cast<const unsigned char*>(UP ? a.gate_up : a.down);
  long tile[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const long in = min((int)blockIdx.x * TILES + t % TILES, units - 1);   // (a tile past the last is computed again and not stored)
    tile[t] = UP ? (long)e * 2 * units + (t / TILES) * units + in : (long)e * units + in;
  }
  const int first = l.chunks * wave / W, last = l.chunks * (wave + 1) / W;
  const Widen<T> widen;
  for (int from = (int)blockIdx.z * ROWS, all = 0x7fffffff; from < all; from += (int)gridDim.z * ROWS) {
    all = pairs_of<W>(a.chosen, a.pairs, e, from, ROWS, rows, counts);
    if (from >= all) return;   // (the same for all threads)
    const int have = min(ROWS, all - from);
    const T* row[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      row[i] = nullptr;
      if (4 * i + g < have) {
        const int p = rows[4 * i + g];
        row[i] = UP ? static_cast<const T*>(a.x) + (long)fast_div((unsigned)p, a.fd_top_k) * a.x_stride : static_cast<const T*>(a.h) + (long)p * a.inter;
      }
    }
    floatx4 sum[NT][RT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) sum[t][r] = (floatx4){0, 0, 0, 0};
    Chunk<T, NT, XL, FL> c;
    if (first < last) c.load(packed, l, per_group, a.zeros, tile, row, first, k, lane);
    for (int chunk = first; chunk < last; ++chunk) {
      const Chunk<T, NT, XL, FL> now = c;
      if (chunk + 1 < last) c.load(packed, l, per_group, a.zeros, tile, row, chunk + 1, k, lane);
      now.template add<RT>(sum, lds[wave], widen, lane);
    }
    floatx4* const part = reinterpret_cast<floatx4*>(lds[wave]);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) part[(t * RT + r) * 64 + lane] = sum[t][r];
    __syncthreads();
    for (int i = (int)threadIdx.x; i < TILES * RT * 64; i += W * 64) {
      const int t = i / (RT * 64), at = i / 64 % RT * 16 + (i & 15), u0 = ((int)blockIdx.x * TILES + t) * 16 + 4 * (i >> 4 & 3);
      if (at >= have || u0 >= units * 16) continue;
      const int p = rows[at];
      floatx4 v[UP ? 2 : 1];
#pragma unroll
      for (int w = 0; w < (UP ? 2 : 1); ++w) {
        v[w] = (floatx4){0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < W; ++u) v[w] += reinterpret_cast<const floatx4*>(lds[u])[i + w * TILES * RT * 64];
        if (__builtin_expect(!is_finite(v[w]), 0)) {
          const T* const x = UP ? static_cast<const T*>(a.x) + (long)fast_div((unsigned)p, a.fd_top_k) * a.x_stride : static_cast<const T*>(a.h) + (long)p * a.inter;
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            const float again = sum_by_weights<T>(packed, l, k, a.group_of(k), a.zeros, x, (UP ? e * 2 * a.inter + w * a.inter : e * a.channels) + u0 + j);
#pragma unroll
            for (int f = 0; f < 4; ++f) v[w][f] = j == f ? again : v[w][f];
          }
        }
      }
      if constexpr (UP) {
        typedef T four __attribute__((ext_vector_type(4)));
        four h;
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = (T)(a.weights[p] * activated(a.act, v[0][j]) * v[UP][j]);
        *reinterpret_cast<four*>(static_cast<T*>(a.h) + (long)p * a.inter + u0) = h;
      } else {
        *reinterpret_cast<floatx4*>(a.parts + (long)p * a.channels + u0) = v[0];
      }
    }
    __syncthreads();
  }
}

// y of a token: its pairs' parts in their order, and the residual.  A thread makes four channels.
template <typename T>
__global__ __launch_bounds__(256) void experts_add_kernel(const ExpertsArgs a) {
  const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4, t = (int)blockIdx.y;
  if (c >= a.channels) return;
  floatx4 v = {0, 0, 0, 0};
  for (int s = 0; s < a.top_k; ++s) {
    const int p = t * a.top_k + s;
    if ((unsigned)a.chosen[p] < (unsigned)a.experts) v += *reinterpret_cast<const floatx4*>(a.parts + (long)p * a.channels + c);
  }
  const long at = (long)t * a.y_stride + c;
#pragma unroll
  for (int j = 0; j < 4; ++j) static_cast<T*>(a.y)[at + j] = (T)(a.res ? v[j] + (float)static_cast<const T*>(a.res)[at + j] : v[j]);
}

template <typename T, bool UP, int TILES, int XL, int W>
hipError_t launch_rows(const ExpertsArgs& a, const W4Layout& l, int blocks, hipStream_t st) {
  const int units = (UP ? a.inter : a.channels) / 16, per_group = a.group_of(UP ? a.channels : a.inter) / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)((units + TILES - 1) / TILES), (unsigned)(a.by_pair ? a.pairs : a.experts), (unsigned)blocks), block(W * 64);
  if (per_group % 4 == 0) hipLaunchKernelGGL((experts_rows_kernel<T, UP, TILES, XL, W, 4>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((experts_rows_kernel<T, UP, TILES, XL, W, 2>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((experts_rows_kernel<T, UP, TILES, XL, W, 1>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const ExpertsArgs& a, hipStream_t st) {
  const W4Layout up = w4_layout(a.experts * 2 * a.inter, a.channels, a.group_of(a.channels), a.zeros != 0);
  const W4Layout down = w4_layout(a.experts * a.channels, a.inter, a.group_of(a.inter), a.zeros != 0);
  const int blocks = a.tokens <= 16 ? 1 : (a.tokens + 15) / 16 < 4 ? (a.tokens + 15) / 16 : 4;
  hipError_t e = a.pairs <= 4 ? launch_rows<T, true, 1, 1, 8>(a, up, 1, st) : launch_rows<T, true, 1, 4, 8>(a, up, blocks, st);
  if (e != hipSuccess) return e;
  e = a.pairs <= 4 ? launch_rows<T, false, 2, 1, 8>(a, down, 1, st) : launch_rows<T, false, 2, 4, 8>(a, down, blocks, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((experts_add_kernel<T>), dim3((unsigned)((a.channels + 1023) / 1024), (unsigned)a.tokens), dim3(256), 0, st, a);
  return hipGetLastError();
}

constexpr int kPairs = 4096;   // of a launch at most
int tokens_at_once(const ExpertsArgs& a) { return a.top_k >= kPairs ? 1 : kPairs / a.top_k; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t experts_workspace_bytes(const ExpertsArgs& a) {
  const size_t pairs = (size_t)(a.tokens < tokens_at_once(a) ? a.tokens : tokens_at_once(a)) * a.top_k;
  return up256(pairs * a.inter * 2) + up256(pairs * a.channels * 4);
}

hipError_t launch_experts(const ExpertsArgs& args, int dtype, hipStream_t st) {
  const int most = tokens_at_once(args);
  for (int first = 0; first < args.tokens; first += most) {
    ExpertsArgs a = args;
    a.tokens = args.tokens - first < most ? args.tokens - first : most;
    a.pairs = a.tokens * a.top_k;
    a.by_pair = a.pairs <= a.experts;
    a.fd_top_k = make_fastdiv((uint32_t)a.top_k);
    const int64_t rows = (int64_t)first * 2;
    a.x = static_cast<const char*>(args.x) + rows * a.x_stride;
    a.y = static_cast<char*>(args.y) + rows * a.y_stride;
    if (a.res) a.res = static_cast<const char*>(args.res) + rows * a.y_stride;
    a.chosen = args.chosen + (size_t)first * a.top_k;
    a.weights = args.weights + (size_t)first * a.top_k;
    a.h = args.workspace;
    a.parts = reinterpret_cast<float*>(static_cast<char*>(args.workspace) + up256((size_t)a.pairs * a.inter * 2));
    if (hipError_t e = dtype == T_F16 ? launch_type<_Float16>(a, st) : launch_type<__bf16>(a, st)) return e;
  }
  return hipSuccess;
}

}  // namespace relay
