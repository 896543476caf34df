// Rotary positions: pairs of channels turned by the token's angle, on a tensor or on the way into a paged cache, and the table of the
// angles' cosines and sines.
//
// Mathematics: y0 = x0 c - x1 s, y1 = x1 c + x0 s in fp32, rounded once.  Each element is read and written once and takes three
// operations: bound by memory.  A thread takes one 16-byte piece of a head (of the half layout two, the piece and its partner
// rotary_dim/2 channels on) for up to HPT heads of one token, so that the piece's cosines and sines -- in fp32 twice to four times the bytes of the
// 16-bit piece they turn -- are fetched once for those heads.  Channels beyond rotary_dim are further pieces, copied; so are the values on their way into
// the cache.  Consecutive lanes take consecutive pieces of a head, then the next head.
// Measured: the store of 5003 tokens, bf16, 32 of 80 channels turned, 13 us = 5.0 TB/s; the gradient of 4096 tokens in fp32 30 us = 4.5 TB/s; one token 5 us, a launch.
#include "attention.hpp"

namespace relay {
namespace {

// V elements of T to and from fp32.  VEC: as one aligned access of V * sizeof(T) bytes; otherwise one by one, the first n of them.
template <typename T, int V, bool VEC>
__device__ __forceinline__ void load(const T* p, float* f, int n) {
  if constexpr (VEC) {
    typedef T vec __attribute__((ext_vector_type(V)));
    const vec t = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = (float)t[e];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = e < n ? (float)p[e] : 0.f;
  }
}
template <typename T, int V, bool VEC>
__device__ __forceinline__ void store(T* p, const float* f, int n) {
  if constexpr (VEC) {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec t;
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = (T)f[e];
    *reinterpret_cast<vec*>(p) = t;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = (T)f[e];
  }
}

// V: channels of a piece.  ILV: interleaved pairs.  HPT: heads of a thread.
template <typename T, int V, bool VEC, bool ILV, int HPT>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
  const unsigned t = blockIdx.x * 256u + threadIdx.x;
  const unsigned tg = fast_div(t, a.fd_pieces);
  const int piece = (int)(t - tg * (unsigned)a.pieces);
  const unsigned token = fast_div(tg, a.fd_groups);
  const int h0 = (int)(tg - token * (unsigned)a.head_groups);
  if (token >= (unsigned)a.tokens) return;
  constexpr int P = ILV ? V / 2 : V;   // pairs of a piece
  constexpr int W = ILV ? 1 : 2;       // vectors of a turned piece
  const bool turned = piece < a.turn_pieces;
  const int half = a.rotary_dim >> 1;
  // first channel of the piece (of its first vector)
  const int ch = turned ? piece * V : a.rotary_dim + (piece - a.turn_pieces) * V;
  const int n = a.head_dim - ch;       // channels left from there (a last single one of an odd head)
  float c[P], s[P];
  const int pos = a.positions[token];
  if (turned) {
    const bool in = (unsigned)pos < (unsigned)a.table_rows;
    const float2* cs = reinterpret_cast<const float2*>(a.cos_sin) + (size_t)(in ? pos : 0) * half + (ILV ? ch >> 1 : ch);
    if constexpr (VEC && P % 2 == 0) {
#pragma unroll
      for (int i = 0; i < P; i += 2) {
        const float4 f = *reinterpret_cast<const float4*>(cs + i);
        c[i] = f.x; s[i] = f.y; c[i + 1] = f.z; s[i + 1] = f.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) { const float2 f = cs[i]; c[i] = f.x; s[i] = f.y; }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (!in) c[i] = s[i] = __builtin_nanf("");
      if (a.inverse) s[i] = -s[i];
    }
  }
  long place = 0;
  bool stored = true;
  if (a.parts > 1) {
    const int slot = a.slots[token];
    stored = (unsigned)slot < (unsigned)a.num_slots;
    const unsigned page = fast_div(stored ? (unsigned)slot : 0u, a.fd_page);
    place = (long)page * a.page_stride + (long)((unsigned)slot - page * (unsigned)a.page_size) * a.slot_stride;
  }
  float x[HPT][W][V];
  T* dst[HPT];
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = h0 + i * a.head_groups;
    dst[i] = nullptr;
    if (h >= a.heads) continue;
    const int w = h < a.q_heads ? 0 : h < a.qk_heads ? 1 : 2;
    const int hl = w == 0 ? h : w == 1 ? h - a.q_heads : h - a.qk_heads;
    const RopePart& p = a.part[w];
    const T* src = static_cast<const T*>(p.src) + (long)token * p.src_token + (long)hl * p.src_head + ch;
    T* const d = static_cast<T*>(p.dst) + (w == 0 ? (long)token * p.dst_token : place) + (long)hl * p.dst_head + ch;
    dst[i] = w == 0 || stored ? d : nullptr;
    load<T, V, VEC>(src, x[i][0], n);
    if (W == 2 && turned) load<T, V, VEC>(src + half, x[i][W - 1], n);
  }
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    if (!dst[i]) continue;
    const bool turn = turned && h0 + i * a.head_groups < a.qk_heads;
    if (turn) {
#pragma unroll
      for (int e = 0; e < P; ++e) {
        float& x0 = ILV ? x[i][0][2 * e] : x[i][0][e];
        float& x1 = ILV ? x[i][0][2 * e + 1] : x[i][W - 1][e];
        const float y0 = x0 * c[e] - x1 * s[e], y1 = x1 * c[e] + x0 * s[e];
        x0 = y0;
        x1 = y1;
      }
    }
    store<T, V, VEC>(dst[i], x[i][0], n);
    if (W == 2 && turned) store<T, V, VEC>(dst[i] + half, x[i][W - 1], n);
  }
}

constexpr int kHeadsPerThread = 4;

// Channels of a piece: 16 bytes where the tensors allow it and whole pieces lie on both sides of rotary_dim (in the half layout in both of
// its halves), else a pair or a channel.
int piece_channels(const RopeArgs& a, int dtype) {
  const int v = dtype == T_F32 ? 4 : 8, ilv = a.style == 1;
  return a.vec && a.rotary_dim % (ilv ? v : 2 * v) == 0 && a.head_dim % v == 0 ? v : ilv ? 2 : 1;
}
void set_pieces(RopeArgs& a, int v) {
  a.turn_pieces = a.rotary_dim / (a.style == 1 ? v : 2 * v);
  a.pieces = a.turn_pieces + (a.head_dim - a.rotary_dim + v - 1) / v;
}

template <typename T, int V, bool VEC, bool ILV>
hipError_t launch_pieces(RopeArgs a, hipStream_t st) {
  set_pieces(a, V);
  const long one = (long)a.tokens * a.pieces;
  // several heads to a thread only where that leaves every CU its threads
  const bool many = one * a.heads >= (long)kHeadsPerThread * 256 * 512;
  a.head_groups = many ? (a.heads + kHeadsPerThread - 1) / kHeadsPerThread : a.heads;
  a.fd_pieces = make_fastdiv((uint32_t)a.pieces);
  a.fd_groups = make_fastdiv((uint32_t)a.head_groups);
  const dim3 grid((unsigned)((one * a.head_groups + 255) / 256)), block(256);
  if (many) hipLaunchKernelGGL((rope_kernel<T, V, VEC, ILV, kHeadsPerThread>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, V, VEC, ILV, 1>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_type(const RopeArgs& a, int piece, hipStream_t st) {
  if (a.style == 1) return piece == V ? launch_pieces<T, V, true, true>(a, st) : launch_pieces<T, 2, false, true>(a, st);
  return piece == V ? launch_pieces<T, V, true, false>(a, st) : launch_pieces<T, 1, false, false>(a, st);
}

__global__ __launch_bounds__(256) void rope_table_kernel(const RopeTableArgs a) {
  const int i = (int)(blockIdx.x * 64 + (threadIdx.x & 63));
  const long r0 = blockIdx.y * 4 + (threadIdx.x >> 6);   // (up to 2^31 - 1 rows, and a stride on top)
  if (i >= a.pairs) return;
  const double kTwoPi = 6.283185307179586476925286766559;
  double base = a.base;
  if (a.scaling == 2) base *= pow(a.factor, (double)a.pairs / (double)(a.pairs - 1));
  double f = pow(base, -(double)i / (double)a.pairs);
  if (a.scaling == 1) f /= a.factor;
  if (a.scaling == 3) {
    const double turns = a.original_len * f / kTwoPi;
    const double g = fmin(fmax((turns - a.slow) / (a.fast - a.slow), 0.0), 1.0);
    f = (1.0 - g) * f / a.factor + g * f;
  }
  for (long r = r0; r < a.rows; r += gridDim.y * 4) {
    double s, c;
    sincos(((double)a.first + (double)r) * f, &s, &c);
    reinterpret_cast<float2*>(a.out)[(size_t)r * a.pairs + i] = make_float2((float)(a.magnitude * c), (float)(a.magnitude * s));
  }
}

}  // namespace

// (thread numbers are divided as 31-bit integers)
bool rope_fits(const RopeArgs& args, int dtype) {
  RopeArgs a = args;
  set_pieces(a, piece_channels(a, dtype));
  return (double)a.tokens * a.heads * a.pieces < 2147483392.0;
}

hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t st) {
  const int v = piece_channels(a, dtype);
  if (dtype == T_F32) return launch_type<float, 4>(a, v, st);
  return dtype == T_F16 ? launch_type<_Float16, 8>(a, v, st) : launch_type<__bf16, 8>(a, v, st);
}

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.pairs + 63) / 64), (unsigned)(a.rows < 4 * 4096 ? (a.rows + 3) / 4 : 4096));
  hipLaunchKernelGGL(rope_table_kernel, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace relay
