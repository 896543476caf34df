// Dense with 4-bit weights and group scales:  y[m,j] = sum_g scale[j,g] sum_{i in g} x[m,i] (code[j,i] - zero[j,g])  and its fused tail.
//
// Codes enter the matrix cores as the exact 16-bit numbers 16 + code: the four bits are moved to the top of the
// mantissa of 16.0, one shift and one and-or for two of them.  With S = sum_{i in g} x[m,i], which a product with ones gives,
//   sum x (code - zero) = sum x (16 + code) - (16 + zero) S
// so the weights are never rounded and a group's scale multiplies an fp32 sum.  The two sides are larger than their difference, so a group's sum is off by up to
// (group + 4) 2^-24 sum |x| (32 + code + zero), where the weights alone would have |code - zero| in that place: beside an output of 16 bits that is small unless codes stand
// close to their zero points.  The tiles of fp16 subtract the zero points from the codes instead, exactly, and pay none of it.
//
// Few rows of x: bound by the codes' bytes.  The waves of a workgroup share 16 units' rows out among them along the reduction, each
// streams its part straight into the A operands (the packed order), and they add up through LDS.
#include <type_traits>

#include "lds_dma.hpp"
#include "w4_common.hpp"

namespace relay {
namespace {

// One sum from the weights themselves, code by code.  Where it is taken: an infinity among x, or values whose sums with the numbers 16 + code leave fp32's range,
// make the two sides of the formula above infinite, and their difference a NaN whatever the weights are.  Such sums, and no others, are not finite, and are
// formed again before the tail; what is read is small beside a launch unless most of x is such values, and one NaN ends it.
template <typename T>
__device__ __forceinline__ float sum_by_weights(const W4Args& a, const W4Layout& l, int m, int j) {
  return sum_by_weights<T>(a.packed, l, a.k, a.group, a.zeros, static_cast<const T*>(a.x) + (long)m * a.x_stride, j);
}

// the tail of one output
template <typename T>
__device__ __forceinline__ void finish(const W4Args& a, int m, int j, float v) {
  if (a.bias) v += a.bias[j];
  if (a.res) v += (float)static_cast<const T*>(a.res)[(long)m * a.y_stride + j];
  if (a.relu) v = v > 0.f ? v : 0.f;
  static_cast<T*>(a.y)[(long)m * a.y_stride + j] = (T)v;
}

// the tail of four units from j on
template <typename T>
__device__ __forceinline__ void finish4(const W4Args& a, int m, int j, floatx4 v) {
  typedef T four __attribute__((ext_vector_type(4)));
  if (!a.wide) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < a.n) finish<T>(a, m, j + e, v[e]);
    return;
  }
  if (j >= a.n) return;
  const long at = (long)m * a.y_stride + j;
  if (a.bias) v += *reinterpret_cast<const floatx4*>(a.bias + j);
  if (a.res) v += __builtin_convertvector(*reinterpret_cast<const four*>(static_cast<const T*>(a.res) + at), floatx4);
  if (a.relu)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] > 0.f ? v[e] : 0.f;
  *reinterpret_cast<four*>(static_cast<T*>(a.y) + at) = __builtin_convertvector(v, four);
}

// Up to MR rows (1 or 4): bound by the codes' bytes, and close behind by the memory pipe, which takes a 16-byte load of a wave in 16 clocks whatever its
// lanes ask for.  So beside the codes' loads there are few others: what a wave needs of x, scales and zero points for SC chunks of its
// part of the reduction comes in whole 16-byte pieces and goes through LDS that only this wave uses.  One row by 32768 x 8192, bf16: 29 to 31 us by box = 4.4 to 4.7 TB/s (31 where this took 29 with a load of
// x and of scales to every chunk, 40 with four of x).
// W waves share the reduction out.  FL: steps of 32 between two applications of the scales, 4 where groups are whole chunks, 2 or 1 where they are not.
template <typename T, int MR, int W, int FL>
__global__ __launch_bounds__(W * 64) void w4_few_kernel(const W4Args a, const W4Layout l, const FastDiv per_group) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  typedef T four __attribute__((ext_vector_type(4)));
  constexpr int SC = MR == 1 ? 8 : 4, XP = SC * 16 * MR, XL = XP / 64, GP = SC * 8;   // 16-byte pieces of x; loads of them; pieces of scales at most
  __shared__ __attribute__((aligned(16))) uintx4 lds[W][XP + GP + GP / 2];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int tile = (int)blockIdx.x, g = lane >> 4, col = lane & 15;
  const unsigned char* base = static_cast<const unsigned char*>(a.packed);
  const int first = l.chunks * wave / W, last = l.chunks * (wave + 1) / W;
  const uintx4* w = reinterpret_cast<const uintx4*>(base) + (size_t)tile * l.chunks * 64 + lane;
  const uintx4* scales = reinterpret_cast<const uintx4*>(base + l.scales_at) + (size_t)tile * l.groups * 2;
  const uintx4* zeros = reinterpret_cast<const uintx4*>(base + l.zeros_at) + (size_t)tile * l.groups;
  uintx4 codes[SC], xv[XL], sv, zv;
  auto group_of = [&](int chunk) { return (int)fast_div((unsigned)(chunk * 4), per_group); };
  auto load_codes = [&](int chunk, int i) { if (chunk < last) codes[i] = w[(size_t)chunk * 64]; };
  auto load_rest = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const int piece = i * 64 + lane, row = piece / (SC * 16), at = chunk * 128 + (piece - row * SC * 16) * 8;
      xv[i] = (uintx4){0, 0, 0, 0};
      if (row < a.m && at < a.k) xv[i] = *reinterpret_cast<const uintx4*>(static_cast<const T*>(a.x) + (long)row * a.x_stride + at);
    }
    const int g0 = group_of(chunk), have = l.groups - g0;
    if (lane < GP && lane < 2 * have) sv = scales[g0 * 2 + lane];
    if (a.zeros && lane < GP / 2 && lane < have) zv = zeros[g0 + lane];
  };
#pragma unroll
  for (int i = 0; i < SC; ++i) load_codes(first + i, i);
  if (first < last) load_rest(first);
  uintx4* const mx = lds[wave];
  const four* const msc = reinterpret_cast<const four*>(mx + XP);             // [group][16 units]
  const unsigned* const mzp = reinterpret_cast<const unsigned*>(mx + XP + GP);
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  const Widen<T> widen;
  const int xrow = (MR == 1 ? 0 : min(col, a.m - 1)) * SC * 16 + g;   // (columns of rows that are not there repeat the last one)
  floatx4 sum = {0, 0, 0, 0};
  for (int c0 = first; c0 < last; c0 += SC) {
#pragma unroll
    for (int i = 0; i < XL; ++i) mx[i * 64 + lane] = xv[i];
    if (lane < GP) mx[XP + lane] = sv;
    if (lane < GP / 2) mx[XP + GP + lane] = zv;
    const int g0 = group_of(c0);
    if (c0 + SC < last) load_rest(c0 + SC);
#pragma unroll
    for (int i = 0; i < SC; ++i) {
      if (c0 + i >= last) break;
#pragma unroll
      for (int f = 0; f < 4 / FL; ++f) {
        floatx4 acc = {0, 0, 0, 0}, xs = {0, 0, 0, 0};
#pragma unroll
        for (int s = f * FL; s < (f + 1) * FL; ++s) {
          const vec xb = __builtin_bit_cast(vec, mx[xrow + i * 16 + s * 4]);
          xs = C::mfma(ones, xb, xs);
          acc = C::mfma(widen(codes[i][s]), xb, acc);
        }
        const int gr = min((int)fast_div((unsigned)((c0 + i) * 4 + f * FL), per_group), l.groups - 1) - g0;
        const four sc = msc[gr * 4 + g];
        const unsigned zp = a.zeros ? mzp[gr * 4 + g] : 0x18181818u;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf((float)sc[e], fmaf(-(float)((zp >> (8 * e)) & 255u), xs[e], acc[e]), sum[e]);
      }
      load_codes(c0 + SC + i, i);
    }
  }
  floatx4* const part = reinterpret_cast<floatx4*>(mx);
  if (col < MR) part[col * 4 + g] = sum;
  __syncthreads();
  // lane: unit lane % 16 of the tile, row lane / 16
  const int t = (int)threadIdx.x, r = t >> 4, j = t & 15;
  if (r >= MR || r >= a.m || tile * 16 + j >= a.n) return;
  float v = 0.f;
#pragma unroll
  for (int u = 0; u < W; ++u) v += reinterpret_cast<const float*>(lds[u])[r * 16 + j];
  if (__builtin_expect(!is_finite(v), 0)) v = sum_by_weights<T>(a, l, r, tile * 16 + j);
  finish<T>(a, r, tile * 16 + j, v);
}

// More rows.  NT tiles of 16 units and RT tiles of 16 rows to a wave, W waves share the reduction out in chunks of 128; the next chunk of
// codes and of x is on its way.  x comes in whole rows of a chunk, 256 bytes to 16 lanes, and is turned into B operands in a piece of LDS
// that only its wave uses: asked for as the operands want it, 64 bytes to a row, sixteen rows of a large power of two apart, it came
// out of few channels of the caches (8192 units by 8192, 16 rows: 20 us, with twice the units to a wave 15; in whole rows 10).
// FL: steps of 32 between two applications of the scales, 4 where groups are whole chunks, 2 or 1 where they are not.
template <typename T, int NT, int RT, int W, int FL>
__global__ __launch_bounds__(W * 64, 2) void w4_rows_kernel(const W4Args a, const W4Layout l, const FastDiv per_group) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  constexpr int XL = 4 * RT;   // loads of x of a chunk, four rows each
  constexpr int XPIECES = RT * 256, SUMS = NT * RT * 64;
  __shared__ __attribute__((aligned(16))) uintx4 lds[W][XPIECES > SUMS ? XPIECES : SUMS];
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
  // load i: row 4 i + lane / 16, 16-byte piece lane % 16 of the chunk
  const T* const x = static_cast<const T*>(a.x) + (long)m0 * a.x_stride + col * 8;
  const int rows = a.m - m0;
  typedef T four __attribute__((ext_vector_type(4)));
  uintx4 codes[NT], xv[XL];
  four sc[4 / FL][NT];
  unsigned zp[4 / FL][NT];
  auto load = [&](int chunk) {
#pragma unroll
    for (int t = 0; t < NT; ++t) codes[t] = w[t][(size_t)chunk * 64];
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
      const int at = min((int)fast_div((unsigned)(chunk * 4 + f * FL), per_group), l.groups - 1) * 16;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        sc[f][t] = *reinterpret_cast<const four*>(scales[t] + at);
        zp[f][t] = a.zeros ? *reinterpret_cast<const unsigned*>(zeros[t] + at) : 0x18181818u;
      }
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      xv[i] = (uintx4){0, 0, 0, 0};
      if (4 * i + g < rows && chunk * 128 + col * 8 < a.k) xv[i] = *reinterpret_cast<const uintx4*>(x + (long)(4 * i + g) * a.x_stride + chunk * 128);
    }
  };
  // (A loop of one turn: unrolled late, it leaves the compiler the addresses of the rows of x to keep; without it they are formed again at each chunk, 8192 units by 8192,
  // 16 rows, 10.1 us and 10.7, 200 rows of 1500 units by 2000 10.5 and 11.3.)
#pragma unroll
  for (int c = first; c < first + 1; ++c)
    if (c < last) load(c);
  uintx4* const mine = lds[wave];
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  const Widen<T> widen;
  floatx4 sum[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[t][r] = (floatx4){0, 0, 0, 0};
  for (int chunk = first; chunk < last; ++chunk) {
#pragma unroll
    for (int i = 0; i < XL; ++i) mine[(4 * i + g) * 16 + (col ^ ((4 * i + g) & 15))] = xv[i];
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
      floatx4 acc[NT][RT], xs[RT];
      const floatx4 none = {0, 0, 0, 0};
#pragma unroll
      for (int s = f * FL; s < (f + 1) * FL; ++s) {
        const bool fresh = s == f * FL;
        vec xb[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          xb[r] = __builtin_bit_cast(vec, mine[(r * 16 + col) * 16 + ((4 * s + g) ^ col)]);
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
          const float z = -(float)((zp[f][t] >> (8 * i)) & 255u), k = (float)sc[f][t][i];
#pragma unroll
          for (int r = 0; r < RT; ++r) sum[t][r][i] = fmaf(k, fmaf(z, xs[r][i], acc[t][r][i]), sum[t][r][i]);
        }
    }
    if (chunk + 1 < last) load(chunk + 1);
  }
  floatx4* const part = reinterpret_cast<floatx4*>(mine);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) part[(t * RT + r) * 64 + lane] = sum[t][r];
  __syncthreads();
  for (int i = (int)threadIdx.x; i < NT * RT * 64; i += W * 64) {
    const int which = i >> 6, ln = i & 63;
    floatx4 v = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < W; ++u) v += reinterpret_cast<const floatx4*>(lds[u])[i];
    const int row = m0 + (which % RT) * 16 + (ln & 15), j0 = (tile0 + which / RT) * 16 + 4 * (ln >> 4);
    if (row >= a.m) continue;
    if (__builtin_expect(!is_finite(v), 0))
#pragma unroll 1
      for (int j = j0; j < min(j0 + 4, a.n); ++j) {
        const float again = sum_by_weights<T>(a, l, row, j);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = j == j0 + e ? again : v[e];
      }
    finish4<T>(a, row, j0, v);
  }
}

// Many rows: a matrix product.  A workgroup makes 128 units of 128 rows, each of its four waves 64 of 64.  Everything goes through LDS, straight from
// memory and two halves of a chunk ahead (64 of the reduction each, one barrier to each): x in a ring of three halves, so that two workgroups fit a CU; codes,
// scales and zero points, which two waves share, in two buffers of a chunk.  A word of codes is widened once for four matrix instructions.  The sums of a group and
// those of all groups are both kept in registers, 64 each.  blockIdx.x runs over the units: workgroups that share rows of x follow each other.
// PARTS 2: eight waves, of which four and four share the reduction out, for launches of so few tiles that a CU has one.
// FL as above.  1500 rows, 8192 units by 4096, fp16: 123 us = 820 TFLOP/s; 1024 rows, 8192 by 8192 152 us = 902;
// 1500 rows in bf16, groups of 32, 197 us = 510: that type has no exact subtraction, and such groups a scale at every step.
template <typename T, int FL, int PARTS>
__global__ __launch_bounds__(256 * PARTS, 2) void w4_tiles_kernel(const W4Args a, const W4Layout l, const FastDiv per_group) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  typedef T four __attribute__((ext_vector_type(4)));
  constexpr int ROWS = 128, TILES = 8, XP = ROWS * 8, CP = TILES * 64, SP = TILES * 8, ZP = TILES * 4;   // 16-byte pieces of a buffer
  constexpr int RING = 3;   // halves of x on their way or in use
  constexpr int XB = RING * XP, WB = CP + SP + ZP, BUF = XB + 2 * WB;
  __shared__ __attribute__((aligned(16))) uintx4 buffers[PARTS][BUF];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) & 3;
  const int part = PARTS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8) : 0;
  const int wu = wave & 1, wr = wave >> 1;
  uintx4* const xl = buffers[part];        // [RING][XP]
  uintx4* const wl = buffers[part] + XB;   // [2][WB]
  const int g = lane >> 4, col = lane & 15;
  const int tile0 = (int)blockIdx.x * TILES, m0 = (int)blockIdx.y * ROWS;
  const char* base = static_cast<const char*>(a.packed);
  // What a wave copies: 32 rows of a half of x; of a chunk the codes of two tiles (a tile past the last is computed again and not stored), wave 0
  // the scales and wave 1 the zero points.  Piece p (16 bytes) of a half row stands at p ^ row / 2 % 8: 16 rows' reads of one piece fall on
  // different banks.
  const T* xs[4];
  int xk[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = (wave * 4 + i) * 64 + lane, row = at >> 3;
    xk[i] = ((at & 7) ^ ((row >> 1) & 7)) * 8;
    xs[i] = static_cast<const T*>(a.x) + (long)min(m0 + row, a.m - 1) * a.x_stride + xk[i];
  }
  const char* ws[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) ws[i] = base + ((size_t)min(tile0 + wave * 2 + i, l.tiles - 1) * l.chunks * 64 + lane) * 16;
  const int ptile = wave == 0 ? lane >> 3 : lane >> 2, piece = wave == 0 ? lane & 7 : lane & 3;   // of scales: two to a group; of zero points: one
  const bool pwanted = wave == 0 || (wave == 1 && a.zeros && lane < ZP);
  const char* const ps = wave == 0 ? base + l.scales_at + ((size_t)min(tile0 + ptile, l.tiles - 1) * l.groups * 2 + piece) * 16
                                   : base + l.zeros_at + ((size_t)min(tile0 + (ptile & 7), l.tiles - 1) * l.groups + piece) * 16;
  const unsigned x_at = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)&buffers[0][0] + (unsigned)(part * BUF * 16);
  const unsigned w_at = x_at + XB * 16;
  auto copy_x = [&](int half, int slot) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (half * 64 + xk[i] < a.k) lds_dma16_at(x_at + (unsigned)(slot * XP * 16 + (wave * 4 + i) * 1024), xs[i] + (long)half * 64);
    if (half * 64 + 64 > a.k)   // pieces that lie behind k: zeros
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (half * 64 + xk[i] >= a.k) xl[slot * XP + (wave * 4 + i) * 64 + lane] = (uintx4){0, 0, 0, 0};
  };
  auto copy_w = [&](int chunk) {
    const unsigned to = w_at + (unsigned)((chunk & 1) * WB * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) lds_dma16_at(to + (unsigned)(wave * 2 + i) * 1024u, ws[i] + (size_t)chunk * 1024);
    if (wave < 2) {
      const int g0 = (int)fast_div((unsigned)(chunk * 4), per_group);
      if (pwanted && (wave == 0 ? g0 + (piece >> 1) : g0 + piece) < l.groups)
        lds_dma16_at(to + (CP + (wave == 0 ? 0 : SP)) * 16, ps + (size_t)g0 * (wave == 0 ? 32 : 16));
    }
  };
  // fp16 subtracts the zero points exactly, two to an instruction, and needs no sums of x; bf16 has no such instruction.
  constexpr bool EXACT = std::is_same<T, _Float16>::value;
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  const Widen<T> widen;
  // this part's chunks first .. last - 1, `turns` at most; its halves end with end - 1
  const int turns = (l.chunks + PARTS - 1) / PARTS, first = part * turns, last = min(l.chunks, first + turns), end = min((a.k + 63) / 64, 2 * last);
  floatx4 sum[4][4], acc[4][4], xsum[EXACT ? 1 : 4];
  halfx2 zero[EXACT ? 4 : 1];   // -(16 + zero point) of this lane's unit of each tile, for the group at hand
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < 4; ++t) sum[t][r] = (floatx4){0, 0, 0, 0};
  if (!a.zeros && lane < ZP) wl[(wave & 1) * WB + CP + SP + lane] = (uintx4){0x18181818u, 0x18181818u, 0x18181818u, 0x18181818u};   // (16 + 8, to stay)
  if (PARTS == 1 || first < last) {
    copy_x(2 * first, 0);
    copy_w(first);
    if (2 * first + 1 < end) copy_x(2 * first + 1, 1);
  }
  // Half `half` has arrived, all waves' copies of it, and no wave reads the buffers any more that are filled next.  A wave's copies return in order: behind
  // those of this half it has asked for the next half of x (four) and, since an even half, for a chunk's codes (two and, wave 0, the scales).
  int slot = 0;   // of the half at hand in the ring
  auto arrive = [&](int half, bool odd) {
    if (half + 2 >= end) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else if (!odd) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
    else if (wave) asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(7) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (half + 2 < end) copy_x(half + 2, slot == 0 ? 2 : slot - 1);
  };
  const floatx4 none = {0, 0, 0, 0};
  auto zeros_of = [&](int chunk, int s) {
    const int gr = min((int)fast_div((unsigned)(chunk * 4 + s), per_group), l.groups - 1) - (int)fast_div((unsigned)(chunk * 4), per_group);
    const unsigned char* const zp = reinterpret_cast<const unsigned char*>(&wl[(chunk & 1) * WB + CP + SP + wu * 16 + gr]) + col;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      zero[t] = __builtin_bit_cast(halfx2, 0xc800c800u + zp[t * 64] * 0x00400040u);   // (n = 16 .. 31 is the half 0x4800 + 64 n)
    }
  };
  auto scales_of = [&](int chunk, int s, int t, float (&k)[4], float (&z)[4]) {
    const int gr = min((int)fast_div((unsigned)(chunk * 4 + s), per_group), l.groups - 1) - (int)fast_div((unsigned)(chunk * 4), per_group);
    const four sc = (reinterpret_cast<const four*>(&wl[(chunk & 1) * WB + CP + wu * 32]) + g)[(t * 4 + gr) * 4];   // [tile][group][4 g ..]
    const unsigned zp = (reinterpret_cast<const unsigned*>(&wl[(chunk & 1) * WB + CP + SP + wu * 16]) + g)[(t * 4 + gr) * 4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = (float)sc[e];
      z[e] = -(float)((zp >> (8 * e)) & 255u);
    }
  };
  auto apply = [&](int chunk, int s) {   // the scales and zero points of step s to the sums of its group so far
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float k[4], z[4];
      scales_of(chunk, s, t, k, z);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[t][r][e] = fmaf(k[e], EXACT ? acc[t][r][e] : fmaf(z[e], xsum[r][e], acc[t][r][e]), sum[t][r][e]);
    }
  };
  auto step = [&](int chunk, int s, bool fresh) {
    const uintx4* const xrow = &xl[slot * XP + (wr * 64 + col) * 8];
    const unsigned* const cl = reinterpret_cast<const unsigned*>(&wl[(chunk & 1) * WB + wu * 256 + lane]) + s;
    vec xb[4];
    if constexpr (EXACT)
      if (fresh) zeros_of(chunk, s);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      xb[r] = __builtin_bit_cast(vec, xrow[r * 128 + ((4 * (s & 1) + g) ^ (col >> 1))]);
      if constexpr (!EXACT) xsum[r] = C::mfma(ones, xb[r], fresh ? none : xsum[r]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      vec wv = widen(cl[t * 256]);
      if constexpr (EXACT) {
        uintx4 u = __builtin_bit_cast(uintx4, wv);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned ue = u[e];
          u[e] = __builtin_bit_cast(unsigned, __builtin_bit_cast(halfx2, ue) + zero[t]);
        }
        wv = __builtin_bit_cast(vec, u);
      }
      if constexpr (FL == 1) {   // (a tile's sums are used up at once and take a fourth of the registers, which reads ahead of them would fill)
        __builtin_amdgcn_sched_barrier(0);
        floatx4 p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = C::mfma(wv, xb[r], none);
        float k[4], z[4];
        scales_of(chunk, s, t, k, z);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[t][r][e] = fmaf(k[e], EXACT ? p[r][e] : fmaf(z[e], xsum[r][e], p[r][e]), sum[t][r][e]);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] = C::mfma(wv, xb[r], fresh ? none : acc[t][r]);
      }
    }
  };
  for (int turn = 0; turn < turns; ++turn) {   // (the same for all waves: each has to meet every barrier)
    const int chunk = first + turn;
    arrive(2 * chunk, false);
    if (PARTS == 1 || chunk < last) {
      if (chunk + 1 < last) copy_w(chunk + 1);
      step(chunk, 0, true);
      step(chunk, 1, FL == 1);
      if (FL == 2) apply(chunk, 1);
      slot = slot == 2 ? 0 : slot + 1;
    }
    if (PARTS > 1 || 2 * chunk + 1 < end) arrive(2 * chunk + 1, true);
    if (2 * chunk + 1 < end) {
      step(chunk, 2, FL <= 2);
      step(chunk, 3, FL == 1);
      if (FL == 2) apply(chunk, 3);
      slot = slot == 2 ? 0 : slot + 1;
    }
    if (FL == 4 && (PARTS == 1 || chunk < last)) apply(chunk, 0);
  }
  if constexpr (PARTS > 1) {
    floatx4* const other = reinterpret_cast<floatx4*>(&buffers[0][0]) + ((int)threadIdx.x & 255);
    static_assert(PARTS == 2 && sizeof(buffers) >= 16 * 256 * 16, "the second part's sums");
    __syncthreads();
    if (part)
#pragma unroll
      for (int i = 0; i < 16; ++i) other[i * 256] = sum[i / 4][i % 4];
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i / 4][i % 4] += other[i * 256];
  }
  unsigned again = 0;   // fours with a sum that is not finite, see sum_by_weights; none where zero points are subtracted exactly
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = m0 + wr * 64 + r * 16 + col;
    if (row >= a.m) continue;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (!EXACT && __builtin_expect(!is_finite(sum[t][r]), 0)) again |= 1u << (r * 4 + t);
      else finish4<T>(a, row, (tile0 + wu * 4 + t) * 16 + 4 * g, sum[t][r]);
    }
  }
  if constexpr (!EXACT)
    for (; again; again &= again - 1) {
      const int i = __builtin_ctz(again), row = m0 + wr * 64 + (i >> 2) * 16 + col, j0 = (tile0 + wu * 4 + (i & 3)) * 16 + 4 * g;
      for (int j = j0; j < min(j0 + 4, a.n); ++j) finish<T>(a, row, j, sum_by_weights<T>(a, l, row, j));
    }
}

// a thread packs one word: eight codes, or one scale, or one zero point
__global__ __launch_bounds__(256) void w4_pack_kernel(int n, int k, int zeros, int turn, W4Layout l, const uint8_t* codes, const uint16_t* scales,
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
      reinterpret_cast<unsigned*>(out)[t] = __builtin_rotateleft32(w, turn);
    } else {
      const size_t u = t - words;
      const int j = (int)(u / ((size_t)l.groups * 16)) * 16 + (int)(u & 15), gr = (int)(u / 16 % l.groups);
      reinterpret_cast<uint16_t*>(out + l.scales_at)[u] = j < n ? scales[(size_t)j * l.groups + gr] : (uint16_t)0;
      if (zeros) (out + l.zeros_at)[u] = j < n ? (uint8_t)(16 + (zps[(size_t)j * l.groups + gr] & 15)) : (uint8_t)0;
    }
  }
}

}  // namespace

hipError_t launch_w4_pack(const W4Args& a, int dtype, const uint8_t* codes, const void* scales, const uint8_t* zeros, void* packed, hipStream_t st) {
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.zeros != 0);
  const size_t items = (size_t)l.tiles * l.chunks * 256 + (size_t)l.tiles * l.groups * 16;
  const unsigned grid = (unsigned)((items + 255) / 256 < 65536 ? (items + 255) / 256 : 65536);
  hipLaunchKernelGGL(w4_pack_kernel, dim3(grid), dim3(256), 0, st, a.n, a.k, a.zeros, dtype == T_F16 ? W4Type<_Float16>::kAt : W4Type<__bf16>::kAt, l, codes, static_cast<const uint16_t*>(scales), zeros,
                     static_cast<unsigned char*>(packed));
  return hipGetLastError();
}

bool w4_fits(const W4Args& a) { return a.m <= 16 * 65535; }

namespace {
template <typename T, int MR, int W>
hipError_t launch_few(const W4Args& a, const W4Layout& l, hipStream_t st) {
  const int per_group = a.group / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)l.tiles), block(W * 64);
  if (per_group % 4 == 0) hipLaunchKernelGGL((w4_few_kernel<T, MR, W, 4>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((w4_few_kernel<T, MR, W, 2>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((w4_few_kernel<T, MR, W, 1>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

template <typename T, int NT, int RT, int W>
hipError_t launch_rows(const W4Args& a, const W4Layout& l, hipStream_t st) {
  const int per_group = a.group / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)((l.tiles + NT - 1) / NT), (unsigned)((a.m + 16 * RT - 1) / (16 * RT))), block(W * 64);
  if (per_group % 4 == 0) hipLaunchKernelGGL((w4_rows_kernel<T, NT, RT, W, 4>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((w4_rows_kernel<T, NT, RT, W, 2>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((w4_rows_kernel<T, NT, RT, W, 1>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

template <typename T, int PARTS>
hipError_t launch_tiles(const W4Args& a, const W4Layout& l, hipStream_t st) {
  const int per_group = a.group / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)((l.tiles + 7) / 8), (unsigned)((a.m + 127) / 128)), block(256 * PARTS);
  if (per_group % 4 == 0) hipLaunchKernelGGL((w4_tiles_kernel<T, 4, PARTS>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((w4_tiles_kernel<T, 2, PARTS>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((w4_tiles_kernel<T, 1, PARTS>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

// More than 16 rows: 32 at a time on the kernel whose waves share the reduction out, or as tiles of 128 x 128, each of which walks the whole reduction: where
// a CU has one of them at most, in two parts at 4 us and 1.25 us a chunk (in one part 1.7 us a chunk), where it has two, 2.35 us a chunk. The other kernel
// takes 2.5 us and 0.67 ns a workgroup and chunk.  Measured, rows / tiles, us, of the two for each call the quicker, unless marked (!):
//   8192 units by 8192, fp16, groups of 128: 64 rows 28 / 84, 128 rows 53 / 85, 256 rows 101 / 85, 512 rows 196 / 88; bf16 the same but for tiles of 89 to 91;
//     groups of 64: 29 / 89, 57 / 90, 110 / 90, 216 / 93, bf16 29 / 103, 58 / 104, 109 / 104, 215 / 105;
//     groups of 32: 40 / 110, 68 / 110, 127 / 111, 245 / 112, bf16 36 / 131, 68 / 131, 128 / 131 (! tiles), 249 / 132
//   4096 units by 4096, groups of 128 / 32: 300 rows 33 / 45, 44 / 58
//   28000 units by 4096, groups of 128: 48 rows 47 / 46 (! rows), 128 rows 92 / 47, 300 rows 213 / 122; groups of 32 64 / 59 (! rows), 125 / 60, 294 / 162
//   1504 units by 2000: 300 rows 11 / 26.
// A chunk of tiles takes up to 1.5 times as long in bf16 and groups of 32 as the rule counts, one of the other kernel up to 1.3 times: where the two are close the
// rule is off by 8 % at most in these.
long tiles_of(const W4Args& a, const W4Layout& l) { return ((l.tiles + 7L) / 8) * ((a.m + 127) / 128); }
bool rows_pay(const W4Args& a, const W4Layout& l) {
  const long tiles = tiles_of(a, l), rows = ((l.tiles + 1L) / 2) * ((a.m + 31) / 32);
  const double t_tiles = tiles <= 256 ? 4 + 1.25 * l.chunks : 2.35 * l.chunks * (double)((tiles + 511) / 512);
  const double t_rows = 2.5 + 0.67e-3 * (double)rows * l.chunks;
  return t_rows < t_tiles;
}

template <typename T>
hipError_t launch_type(const W4Args& a, const W4Layout& l, hipStream_t st) {
  // Up to four rows on the kernel for few (us, it / the other at 4 rows: 4096 units by 4096 5.2 / 5.4, 8192 by 8192 10.7 / 11.5, in groups of 32 13.3 / 13.4; 32768 by 4096 19.5 / 19.8,
  // in groups of 32 23 / 30; 32768 by 8192 35 / 29, in groups of 32 42 / 49).  Up to 16, two tiles of units to a workgroup where that leaves every CU one (us, one / two
  // tiles: 4096 units by 8192, 16 rows 10.6 / 11.6, 4112 by 8192 12.5 / 11.7, 8192 by 4096 8.8 / 8.6, 6 rows 7.1 / 8.0, 28000 by 4096 22.8 / 20.2, 6 rows 19 / 17.7).
  if (a.m == 1) return launch_few<T, 1, 8>(a, l, st);
  if (a.m <= 4) return launch_few<T, 4, 8>(a, l, st);
  if (a.m <= 16) return l.tiles <= 256 ? launch_rows<T, 1, 1, 8>(a, l, st) : launch_rows<T, 2, 1, 8>(a, l, st);
  if (rows_pay(a, l)) return launch_rows<T, 2, 2, 8>(a, l, st);
  return tiles_of(a, l) <= 256 ? launch_tiles<T, 2>(a, l, st) : launch_tiles<T, 1>(a, l, st);
}
}  // namespace

hipError_t launch_w4(const W4Args& args, int dtype, hipStream_t st) {
  W4Args a = args;
  a.wide = a.n % 4 == 0 && a.y_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.res)) % 8 == 0 &&
           reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.zeros != 0);
  return dtype == T_F16 ? launch_type<_Float16>(a, l, st) : launch_type<__bf16>(a, l, st);
}

}  // namespace relay
