// The experts of a mixture with 4-bit weights for a few tokens:  h = act(gate x) (up x),  y = sum over a token's experts of weight down h.
//
// A pair is a token and one of the experts it has chosen; pairs of one expert share its codes, which are most of what there is to read.  The first
// launch makes h of every pair; the second y, of few pairs directly (a workgroup adds up what the experts make of 16 channels), of more through a pair's parts in memory, which a third adds
// up.  h is rounded to 16 bits, an operand of the matrix cores.  A router's weight is applied to its pair's part of y, in fp32: within h a small one took fp16's bits (a weight of
// 0.002 at an h of 1e-3: 1 % of the part).  A wave streams the codes of two tiles of 16 units through its registers and knows nothing of other waves: with the
// reduction shared out over eight, 64 tokens on 128 experts took 343 us for the first product and 504 for the second, now 115 to 123 and 67 to 70 (4.4 to 4.8 and 4.0 to 4.2 TB/s).  Many rows to an expert: tiles, below.
// One token on 8 experts, 4096 channels and 1024 beside them, fp16: 19 us, 12 and 8, two chains of loads (the 50 MB take 10).  500 tokens on 32 experts, 2048 and 1408: 96 us, plan 5, tiles 58 and 35, sum 5:
// 47 blocks of 43 rows on the mean.  Vector and matrix work are 65 % of the clocks, the rest the start and end of a tile and the chain within a chunk (without the rows' copies 89 us, without the codes' loads 97, without
// both 86); 1034 tiles on 768 places leave a second round short.
// Codes become operands as in the dense kernels (16 + code, the sums of x taking the zero points out).
#include <type_traits>

#include "decoder_ops.hpp"
#include "lds_dma.hpp"
#include "row_piece.hpp"
#include "w4_common.hpp"

namespace relay {
namespace {

constexpr int kBlock = 64;   // pairs of one expert in a tile

// The pairs that name expert e, of those from `from` on the first `most`, into this wave's rows; how many there are in all, and which is the first.
struct Found { int all, first; };
__device__ __forceinline__ Found pairs_of(const int32_t* chosen, int pairs, int e, int from, int most, int* rows, int lane) {
  Found f{0, pairs};
  for (int p0 = 0; p0 < pairs; p0 += 512) {   // (eight loads on their way: one by one each waits for its own)
    int named[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) named[i] = chosen[min(p0 + i * 64 + lane, pairs - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = p0 + i * 64;
      const bool mine = p + lane < pairs && named[i] == e;
      const unsigned long long set = __ballot(mine);
      if (!set) continue;
      if (!f.all) f.first = p + __builtin_ctzll(set);
      const int at = f.all + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0u)) - from;
      if (mine && at >= 0 && at < most) rows[at] = p + lane;
      f.all += __builtin_popcountll(set);
    }
  }
  return f;
}

// What a wave holds of a chunk of 128 of the reduction: codes of NT tiles of 16 units; XL loads of x, four rows each; scales and zero points, which come in whole 16-byte
// pieces and go through LDS with x (a load of a wave takes the memory pipe 16 clocks whatever its lanes ask for).
// FL: steps of 32 between two applications of the scales, 4 where groups are whole chunks, 2 or 1 where they are not.
// All loads are made, of something that is there: which of them return when is then known ahead, and a wait is for those of its chunk alone.
template <typename T, int NT, int XL, int FL>
struct Chunk {
  typedef T four __attribute__((ext_vector_type(4)));
  static constexpr int PG = 4 / FL, PIECES = XL * 64 + NT * PG * 3;   // groups of a chunk at most; 16-byte pieces of LDS
  uintx4 codes[NT], x[XL], params;
  // One place of a stack of units.
  struct Where {
    const uintx4* codes[NT];   // of the tiles' first chunk (the same for all lanes)
    const uintx4* params;      // this lane's piece of the scales (of the zero points) of the tiles' first group
    int step, half;            // pieces from group to group; of scales
    const T* row[XL];          // this lane's rows
    __device__ __forceinline__ void set(const unsigned char* packed, const W4Layout& l, bool zeros, const long (&tile)[NT], int lane) {
#pragma unroll
      for (int t = 0; t < NT; ++t) codes[t] = reinterpret_cast<const uintx4*>(packed) + (size_t)tile[t] * l.chunks * 64;
      // lanes: [tile][group] scales of two pieces, then [tile][group] zero points of one
      const int which = min(lane, NT * PG * 3 - 1), z = which - NT * PG * 2;
      long at = tile[0];
#pragma unroll
      for (int t = 1; t < NT; ++t)
        if ((z < 0 ? which / (2 * PG) : z / PG) == t) at = tile[t];
      const bool zp = z >= 0 && zeros;
      step = zp ? 1 : 2;
      half = z < 0 ? (which & 1) : 0;
      params = reinterpret_cast<const uintx4*>(packed + (zp ? l.zeros_at : l.scales_at)) + (size_t)at * l.groups * step + half;
      group = z < 0 ? which % (2 * PG) / 2 : z % PG;
    }
    int group;                 // this lane's of a chunk's groups
  };
  __device__ __forceinline__ void load_codes(const Where& w, const W4Layout& l, const FastDiv& per_group, int chunk, int lane) {
#pragma unroll
    for (int t = 0; t < NT; ++t) codes[t] = (w.codes[t] + (size_t)chunk * 64)[(unsigned)lane];
    params = w.params[(size_t)min((int)fast_div((unsigned)(chunk * 4), per_group) + w.group, l.groups - 1) * w.step];
  }
  __device__ __forceinline__ void load_x(const Where& w, int chunk, int k, int lane) {
    const int at = row_piece(chunk, lane & 15, k);   // (what lies past k is taken as zeros)
#pragma unroll
    for (int i = 0; i < XL; ++i) x[i] = *reinterpret_cast<const uintx4*>(w.row[i] + at);
  }
  // sums += the chunk's part; mine: PIECES of LDS of this wave
  __device__ __forceinline__ void add(floatx4 (&sum)[NT], uintx4* mine, const W4Layout& l, const FastDiv& per_group, bool zeros, const Widen<T>& widen, int chunk, int k, int lane) const {
    typedef W4Type<T> C;
    typedef typename C::vec vec;
    const int g = lane >> 4, col = lane & 15;
    const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
    const floatx4 none = {0, 0, 0, 0};
    const bool there = chunk * 128 + col * 8 < k;   // (what lies past k: zeros)
#pragma unroll
    for (int i = 0; i < XL; ++i) mine[(4 * i + g) * 16 + (col ^ ((4 * i + g) & 15))] = there ? x[i] : (uintx4){0, 0, 0, 0};
    if (lane < NT * PG * 3) mine[XL * 64 + lane] = params;
    const four* const scales = reinterpret_cast<const four*>(mine + XL * 64);
    const unsigned* const zps = reinterpret_cast<const unsigned*>(mine + XL * 64 + NT * PG * 2);
#pragma unroll
    for (int f = 0; f < PG; ++f) {
      floatx4 acc[NT], xs;
#pragma unroll
      for (int s = f * FL; s < (f + 1) * FL; ++s) {
        const bool fresh = s == f * FL;
        const int at = col & (4 * XL - 1);   // (of fewer rows than columns: those behind repeat them)
        const vec xb = __builtin_bit_cast(vec, mine[at * 16 + ((4 * s + g) ^ (at & 15))]);
        xs = C::mfma(ones, xb, fresh ? none : xs);
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = C::mfma(widen(codes[t][s]), xb, fresh ? none : acc[t]);
      }
      // (the group of step f * FL, counted from the chunk's first)
      const int gr = PG == 1 ? 0 : min((int)fast_div((unsigned)(chunk * 4 + f * FL), per_group), l.groups - 1) - (int)fast_div((unsigned)(chunk * 4), per_group);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const four sc = scales[(t * PG + gr) * 4 + g];
        const unsigned zp = zeros ? zps[(t * PG + gr) * 4 + g] : 0x18181818u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float z = -(float)((zp >> (8 * i)) & 255u), kf = (float)sc[i];
          sum[t][i] = fmaf(kf, fmaf(z, xs[i], acc[t][i]), sum[t][i]);
        }
      }
    }
  }
};

__device__ __forceinline__ float activated(int act, float v) {
  return act == A_SILU ? v / (1.f + expf(-v)) : 0.5f * v * erfcf(v * -0.70710678118654752440f);   // (1 + erf(v) is erfc(-v), without the difference)
}

// sums += chunks first .. last - 1 of the tiles, D of them on their way: c holds the first D.
template <int D, typename T, int NT, int XL, int FL>
__device__ __forceinline__ void walk(floatx4 (&sum)[NT], Chunk<T, NT, XL, FL> (&c)[D], const typename Chunk<T, NT, XL, FL>::Where& w, const W4Layout& l, const FastDiv& per_group, bool zeros,
                                     int first, int last, int k, uintx4* mine, const Widen<T>& widen, int lane) {
  int chunk = first;
  for (; chunk + D < last; chunk += D) {
#pragma unroll
    for (int i = 0; i < D; ++i) {
      c[i].add(sum, mine, l, per_group, zeros, widen, chunk + i, k, lane);
      c[i].load_codes(w, l, per_group, min(chunk + i + D, last - 1), lane);
      c[i].load_x(w, min(chunk + i + D, last - 1), k, lane);
      __builtin_amdgcn_sched_barrier(0);   // (two chunks' sums side by side take twice the registers)
    }
  }
#pragma unroll
  for (int i = 0; i < D; ++i) {
    if (chunk + i < last) c[i].add(sum, mine, l, per_group, zeros, widen, chunk + i, k, lane);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A wave: n times two tiles of 16 units of an expert (UP: of its gates and the ones beside them, for h; not UP: for a pair's part of y, in fp32) for blocks of up to
// XL * 4 of the expert's pairs.  KS > 1: that many waves share the reduction of the same two tiles out (n = 1).  Waves know nothing of each other otherwise.
template <typename T, bool UP, int XL, int KS, int D, int W, int FL>
__global__ __launch_bounds__(W * 64, 2) void experts_rows_kernel(const ExpertsArgs a, const W4Layout l, const FastDiv per_group, const int n) {
  typedef Chunk<T, 2, XL, FL> Held;
  constexpr int ROWS = XL * 4, SUMS = 2 * 64, LDS = Held::PIECES > SUMS ? Held::PIECES : SUMS, PER = UP ? 1 : 2;
  __shared__ __attribute__((aligned(16))) uintx4 lds[W][LDS];
  __shared__ int rows_of[W][ROWS];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4;
  const int e = a.by_pair ? a.chosen[blockIdx.y] : (int)blockIdx.y;
  if ((unsigned)e >= (unsigned)a.experts) return;
  const int k = UP ? a.channels : a.inter, units = (UP ? a.inter : a.channels) / 16;
  const unsigned char* const packed = static_cast<const unsigned char*>(UP ? a.gate_up : a.down);
  const int tile0 = ((int)blockIdx.x * (W / KS) + wave / KS) * PER * n;   // the first of this wave's outputs
  if (KS == 1 && tile0 >= units) return;
  // (a tile past the last: the last again, not stored)
  const long base = UP ? (long)e * 2 * units : (long)e * units;
  const int part = wave % KS, first = l.chunks * part / KS, last = l.chunks * (part + 1) / KS, many = KS > 1 ? 1 : min(n, (units - tile0 + PER - 1) / PER);
  const Widen<T> widen;
  uintx4* const mine = lds[wave];
  int* const rows = rows_of[wave];
  auto x_of = [&](int p) { return UP ? static_cast<const T*>(a.x) + (long)fast_div((unsigned)p, a.fd_top_k) * a.x_stride : static_cast<const T*>(a.h) + (long)p * a.inter; };
  typename Held::Where where;
  Held c[D];
  auto at_tile = [&](int i) {
    const int t = min(tile0 + i * PER, units - 1);
    const long tile[2] = {base + t, base + (UP ? t + units : min(t + 1, units - 1))};
    where.set(packed, l, a.zeros, tile, lane);
#pragma unroll
    for (int j = 0; j < D; ++j) c[j].load_codes(where, l, per_group, max(min(first + j, last - 1), 0), lane);
  };
  auto load_x = [&]() {
#pragma unroll
    for (int j = 0; j < D; ++j) c[j].load_x(where, max(min(first + j, last - 1), 0), k, lane);
  };
  for (int from = 0;; from += ROWS) {
    at_tile(0);   // (on its way while the rows are looked up)
    const Found found = pairs_of(a.chosen, a.pairs, e, from, ROWS, rows, lane);
    if (from >= found.all || (a.by_pair && found.first != (int)blockIdx.y)) return;   // (an expert's first pair stands for it; the same for all waves)
    const int have = min(ROWS, found.all - from);
#pragma unroll
    for (int i = 0; i < XL; ++i) where.row[i] = x_of(rows[min(4 * i + g, have - 1)]);   // (rows that are not there repeat the last one)
    load_x();
    for (int i = 0; i < many; ++i) {
      floatx4 sum[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      if (first < last) walk<D, T, 2, XL, FL>(sum, c, where, l, per_group, a.zeros, first, last, k, mine, widen, lane);
#pragma unroll
      for (int t = 0; t < 2; ++t) reinterpret_cast<floatx4*>(mine)[t * 64 + lane] = sum[t];
      if (i + 1 < many) {
        at_tile(i + 1);
        load_x();
      }
      if (KS > 1) __syncthreads();
      // four units of a pair: to a lane in turn of the KS waves
#pragma unroll 1
      for (int j = KS > 1 ? (wave % KS) * 64 + lane : lane; j < PER * 64; j += KS * 64) {
        const int t = j / 64, at = j & 15, tl = tile0 + i * PER + t;
        if (at >= have || tl >= units) continue;
        floatx4 v[UP ? 2 : 1];
        const int p = rows[at], u0 = tl * 16 + 4 * (j >> 4 & 3);
#pragma unroll
        for (int w = 0; w < (UP ? 2 : 1); ++w) {
          v[w] = (floatx4){0, 0, 0, 0};
#pragma unroll
          for (int u = 0; u < KS; ++u) v[w] += reinterpret_cast<const floatx4*>(lds[wave / KS * KS + u])[j + w * 64];
          if (__builtin_expect(!is_finite(v[w]), 0))
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              const float again = sum_by_weights<T>(packed, l, k, a.group_of(k), a.zeros, x_of(p), (UP ? (2 * e + w) * a.inter : e * a.channels) + u0 + q);
#pragma unroll
              for (int f = 0; f < 4; ++f) v[w][f] = q == f ? again : v[w][f];
            }
        }
        if constexpr (UP) {
          typedef T four __attribute__((ext_vector_type(4)));
          four h;
#pragma unroll
          for (int q = 0; q < 4; ++q) h[q] = (T)(activated(a.act, v[0][q]) * v[1][q]);
          *reinterpret_cast<four*>(static_cast<T*>(a.h) + (long)p * a.inter + u0) = h;
        } else {
          *reinterpret_cast<floatx4*>(a.parts + (long)p * a.channels + u0) = v[0];
        }
      }
      if (KS > 1) __syncthreads();
    }
    if (from + ROWS >= found.all) return;
  }
}

// Pairs by their experts, for the tiles: sorted, and the blocks of up to 64 of them that one expert has (in a.blocks: expert, first place, how many; behind the last an expert of -1).  One workgroup.
// The order of an expert's pairs is of no consequence: a row of a product does not hang on its place.
constexpr int kPlanThreads = 1024;
static_assert(kRouteExperts <= kPlanThreads, "an expert to a thread");
__global__ __launch_bounds__(kPlanThreads) void experts_plan_kernel(const ExpertsArgs a) {
  __shared__ int count[kPlanThreads], sums[2][kPlanThreads / 64];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  count[tid] = 0;
  __syncthreads();
  for (int p = tid; p < a.pairs; p += kPlanThreads) {
    const int e = a.chosen[p];
    if ((unsigned)e < (unsigned)a.experts) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  const int n = count[tid], blocks = (n + kBlock - 1) / kBlock;
  int pairs_to = n, blocks_to = blocks;   // up to and with this expert's
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(pairs_to, d), q = __shfl_up(blocks_to, d);
    if (lane >= d) pairs_to += o, blocks_to += q;
  }
  if (lane == 63) sums[0][wave] = pairs_to, sums[1][wave] = blocks_to;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int u = 0; u < kPlanThreads / 64; ++u) {
    if (u < wave) pairs_to += sums[0][u], blocks_to += sums[1][u];
    all += sums[1][u];
  }
  count[tid] = pairs_to - n;   // where its next pair goes
  for (int i = 0; i < blocks; ++i) {
    int* const b = a.blocks + (blocks_to - blocks + i) * 3;
    b[0] = tid;
    b[1] = pairs_to - n + i * kBlock;
    b[2] = min(kBlock, n - i * kBlock);
  }
  for (int i = all + tid; i < a.most_blocks; i += kPlanThreads) a.blocks[i * 3] = -1;
  __syncthreads();
  for (int p = tid; p < a.pairs; p += kPlanThreads) {
    const int e = a.chosen[p];
    if ((unsigned)e < (unsigned)a.experts) a.sorted[atomicAdd(&count[e], 1)] = p;
  }
}

// Many rows to an expert: a matrix product of 64 pairs by 64 units of h (64 gates and the 64 beside them) or 128 channels of a pair's part of y.  The rows go through LDS, straight from memory and a
// chunk ahead, for all four waves; a wave widens the codes of its two tiles once for all of them, and leaves out the sixteens of rows that are not there.
// fp16 subtracts the zero points from the codes, exactly; bf16 has no such instruction, and takes them out with the sums of x.
template <typename T, bool UP, int FL>
__global__ __launch_bounds__(256, (std::is_same<T, _Float16>::value ? 3 : 2)) void experts_tiles_kernel(const ExpertsArgs a, const W4Layout l, const FastDiv per_group) {
  typedef W4Type<T> C;
  typedef typename C::vec vec;
  typedef T four __attribute__((ext_vector_type(4)));
  constexpr bool EXACT = std::is_same<T, _Float16>::value;
  constexpr int ROWS = kBlock, RT = 4, W = 4, NT = 2, PG = 4 / FL, XP = ROWS * 16, PP = NT * PG * 3;   // 16-byte pieces of a chunk of rows; of a wave's scales and zero points
  __shared__ __attribute__((aligned(16))) uintx4 xs_lds[2][XP];
  __shared__ __attribute__((aligned(16))) uintx4 params_lds[W][2][PP];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
  const int* const block = a.blocks + (int)blockIdx.y * 3;
  const int e = block[0], have = block[2], tiles = (have + 15) / 16;
  if (e < 0) return;
  const int* const rows = a.sorted + block[1];
  const int k = UP ? a.channels : a.inter, units = (UP ? a.inter : a.channels) / 16;
  const unsigned char* const packed = static_cast<const unsigned char*>(UP ? a.gate_up : a.down);
  const int tile0 = UP ? (int)blockIdx.x * W + wave : ((int)blockIdx.x * W + wave) * 2;
  const long base = UP ? (long)e * 2 * units : (long)e * units;
  // (a tile past the last: the last again, not stored)
  const long tile[2] = {base + min(tile0, units - 1), base + (UP ? min(tile0, units - 1) + units : min(tile0 + 1, units - 1))};
  typedef Chunk<T, NT, 1, FL> Held;
  typename Held::Where where;
  where.set(packed, l, a.zeros, tile, lane);
  const Widen<T> widen;
  const vec ones = __builtin_bit_cast(vec, (uintx4){C::kOne, C::kOne, C::kOne, C::kOne});
  const floatx4 none = {0, 0, 0, 0};
  const unsigned x_at = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)&xs_lds[0][0];
  auto x_of = [&](int p) { return UP ? static_cast<const T*>(a.x) + (long)fast_div((unsigned)p, a.fd_top_k) * a.x_stride : static_cast<const T*>(a.h) + (long)p * a.inter; };
  // This wave copies rows 16 wave .. 16 wave + 15 of a chunk, four to an instruction; piece p of a row stands at p ^ row % 16: sixteen rows' reads of one piece fall on different
  // banks.  (Rows that are not there repeat the last one.)
  const T* src[4];
  int at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = wave * 16 + 4 * i + g;
    at[i] = (col ^ (row & 15)) * 8;
    src[i] = x_of(rows[min(row, have - 1)]) + at[i];
  }
  auto copy = [&](int chunk) {
    if (wave >= tiles) return;
    const int buffer = chunk & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (chunk * 128 + at[i] < k) lds_dma16_at(x_at + (unsigned)((buffer * XP + (wave * 16 + 4 * i) * 16) * 16), src[i] + chunk * 128);
    if (chunk * 128 + 128 > k)   // pieces that lie behind k: zeros
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (chunk * 128 + at[i] >= k) xs_lds[buffer][(wave * 16 + 4 * i) * 16 + lane] = (uintx4){0, 0, 0, 0};
  };
  floatx4 sum[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[t][r] = none;
  Held c[2];
  c[0].load_codes(where, l, per_group, 0, lane);
  copy(0);
  c[1].load_codes(where, l, per_group, min(1, l.chunks - 1), lane);
  auto turn = [&](Held& now, int chunk) {
    // Behind the rows of this chunk a wave has asked for one chunk's codes: two loads, and one of scales.
    asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // (What was loaded for this chunk is taken before more is asked for: the compiler does not count the copies, and a wait for the codes would be one for copies just begun.)
    uintx4* const mine = params_lds[wave][chunk & 1];
    if (lane < PP) mine[lane] = now.params;
    uintx4 codes[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      codes[t] = now.codes[t];
      asm volatile("" : "+v"(codes[t]));
    }
    if (chunk + 1 < l.chunks) copy(chunk + 1);
    now.load_codes(where, l, per_group, min(chunk + 2, l.chunks - 1), lane);
    const uintx4* const xl = xs_lds[chunk & 1];
    const four* const scales = reinterpret_cast<const four*>(mine);
    const unsigned* const zps = reinterpret_cast<const unsigned*>(mine + NT * PG * 2);
#pragma unroll
    for (int f = 0; f < PG; ++f) {
      const int gr = PG == 1 ? 0 : min((int)fast_div((unsigned)(chunk * 4 + f * FL), per_group), l.groups - 1) - (int)fast_div((unsigned)(chunk * 4), per_group);
      vec wv[NT][FL];
      float sc[NT][4], zp[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const four s4 = scales[(t * PG + gr) * 4 + g];
        const unsigned z4 = a.zeros ? zps[(t * PG + gr) * 4 + g] : 0x18181818u;
        const unsigned zc = a.zeros ? reinterpret_cast<const unsigned char*>(zps + (t * PG + gr) * 4)[col] : 0x18u;   // of the unit whose codes this lane holds
        const halfx2 minus = __builtin_bit_cast(halfx2, 0xc800c800u + zc * 0x00400040u);                              // (n = 16 .. 31 is the half 0x4800 + 64 n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[t][i] = (float)s4[i];
          zp[t][i] = -(float)((z4 >> (8 * i)) & 255u);
        }
#pragma unroll
        for (int s = 0; s < FL; ++s) {
          wv[t][s] = widen(codes[t][f * FL + s]);
          if constexpr (EXACT) {
            uintx4 u = __builtin_bit_cast(uintx4, wv[t][s]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const unsigned uq = u[q];
              u[q] = __builtin_bit_cast(unsigned, __builtin_bit_cast(halfx2, uq) + minus);
            }
            wv[t][s] = __builtin_bit_cast(vec, u);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r >= tiles) break;
        floatx4 acc[NT], xs = none;
#pragma unroll
        for (int s = 0; s < FL; ++s) {
          const vec xb = __builtin_bit_cast(vec, xl[(r * 16 + col) * 16 + ((4 * (f * FL + s) + g) ^ col)]);
          if constexpr (!EXACT) xs = C::mfma(ones, xb, xs);
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t] = C::mfma(wv[t][s], xb, s ? acc[t] : none);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[t][r][i] = fmaf(sc[t][i], EXACT ? acc[t][i] : fmaf(zp[t][i], xs[i], acc[t][i]), sum[t][r][i]);
      }
    }
  };
  for (int chunk = 0; chunk < l.chunks; chunk += 2) {
    turn(c[0], chunk);
    if (chunk + 1 < l.chunks) turn(c[1], chunk + 1);
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = r * 16 + col;
    if (row >= have) continue;
    const int p = rows[row];
    if constexpr (UP) {
      if (tile0 >= units) continue;
      four h;
      floatx4 v[2] = {sum[0][r], sum[1][r]};
      if constexpr (!EXACT)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (__builtin_expect(!is_finite(v[w]), 0))
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              const float again = sum_by_weights<T>(packed, l, k, a.group_of(k), a.zeros, x_of(p), (2 * e + w) * a.inter + tile0 * 16 + 4 * g + q);
#pragma unroll
              for (int f = 0; f < 4; ++f) v[w][f] = q == f ? again : v[w][f];
            }
#pragma unroll
      for (int q = 0; q < 4; ++q) h[q] = (T)(activated(a.act, v[0][q]) * v[1][q]);
      *reinterpret_cast<four*>(static_cast<T*>(a.h) + (long)p * a.inter + tile0 * 16 + 4 * g) = h;
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (tile0 + t >= units) continue;
        floatx4 v = sum[t][r];
        if constexpr (!EXACT)
          if (__builtin_expect(!is_finite(v), 0))
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              const float again = sum_by_weights<T>(packed, l, k, a.group_of(k), a.zeros, x_of(p), e * a.channels + (tile0 + t) * 16 + 4 * g + q);
#pragma unroll
              for (int f = 0; f < 4; ++f) v[f] = q == f ? again : v[f];
            }
        *reinterpret_cast<floatx4*>(a.parts + (long)p * a.channels + (tile0 + t) * 16 + 4 * g) = v;
      }
    }
  }
}

// y of up to kJoined pairs at once: a workgroup makes 16 channels of all tokens.  Its waves take the chosen experts in turn (several share one's reduction where there are fewer experts than waves), leave
// each pair's part in LDS, and add a token's up in the order of its choices.
constexpr int kJoined = 16, kJoinWaves = 8;
template <typename T, int XL, int FL>
__global__ __launch_bounds__(kJoinWaves * 64, 2) void experts_join_kernel(const ExpertsArgs a, const W4Layout l, const FastDiv per_group) {
  typedef Chunk<T, 1, XL, FL> Held;
  constexpr int D = 2, W = kJoinWaves, ROWS = XL * 4;
  __shared__ __attribute__((aligned(16))) uintx4 lds[W][Held::PIECES];
  __shared__ __attribute__((aligned(16))) floatx4 parts[W * kJoined][4];   // [share of the reduction][pair]
  __shared__ int rows_of[W][kJoined];
  __shared__ float weight_of[kJoined];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, tile = (int)blockIdx.x;
  const unsigned char* const packed = static_cast<const unsigned char*>(a.down);
  const T* const h = static_cast<const T*>(a.h);
  const int named = lane < a.pairs ? a.chosen[lane] : -1;
  const float weight = lane < a.pairs ? a.weights[lane] : 0.f;
  const unsigned long long valid = __ballot((unsigned)named < (unsigned)a.experts);
  int many = 0;
  for (unsigned long long left = valid; left; ++many) left &= ~__ballot(named == __builtin_amdgcn_readlane(named, __builtin_ctzll(left)));
  const int shares = many >= W ? 1 : many >= W / 2 ? 2 : many >= W / 4 ? 4 : W;
  const Widen<T> widen;
  uintx4* const mine = lds[wave];
  int* const rows = rows_of[wave];
  unsigned long long left = valid;
  for (int unit = 0; left; ++unit) {
    const int e = __builtin_amdgcn_readlane(named, __builtin_ctzll(left));
    const unsigned long long set = __ballot(named == e);
    left &= ~set;
    const int turn = (wave - unit * shares % W + W) % W;   // this wave's share of the unit, if it has one
    if (turn >= shares) continue;
    const int have = __builtin_popcountll(set), first = l.chunks * turn / shares, last = l.chunks * (turn + 1) / shares;
    if (set >> lane & 1) rows[(int)__builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0u))] = lane;
    typename Held::Where where;
    const long at[1] = {(long)e * (a.channels / 16) + tile};
    where.set(packed, l, a.zeros, at, lane);
    for (int from = 0; from < have; from += ROWS) {
      floatx4 sum[1] = {{0, 0, 0, 0}};
#pragma unroll
      for (int i = 0; i < XL; ++i) where.row[i] = h + (long)rows[min(from + 4 * i + g, have - 1)] * a.inter;   // (rows that are not there repeat the last one)
      if (first < last) {
        Held c[D];
#pragma unroll
        for (int j = 0; j < D; ++j) c[j].load_codes(where, l, per_group, min(first + j, last - 1), lane);
#pragma unroll
        for (int j = 0; j < D; ++j) c[j].load_x(where, min(first + j, last - 1), a.inter, lane);
        walk<D, T, 1, XL, FL>(sum, c, where, l, per_group, a.zeros, first, last, a.inter, mine, widen, lane);
      }
      const int row = from + (lane & 15);
      if ((lane & 15) < ROWS && row < have) parts[turn * kJoined + rows[row]][g] = sum[0];
    }
  }
  if (wave == 0 && lane < kJoined) weight_of[lane] = weight;
  __syncthreads();
  for (int i = (int)threadIdx.x; i < a.tokens * 16; i += W * 64) {
    const int t = i >> 4, j = i & 15;
    float v = 0.f;
    for (int p = t * a.top_k; p < (t + 1) * a.top_k; ++p) {
      if (!(valid >> p & 1)) continue;
      float part = 0.f, w = weight_of[p];
      for (int u = 0; u < shares; ++u) part += reinterpret_cast<const float*>(parts[u * kJoined + p])[j];
      asm volatile("" : "+v"(w));   // (asked for with the part: behind the branch it would be a read of its own)
      if (__builtin_expect(!is_finite(part), 0))
        part = sum_by_weights<T>(packed, l, a.inter, a.group_of(a.inter), a.zeros, h + (long)p * a.inter, a.chosen[p] * a.channels + tile * 16 + j);
      v = fmaf(w, part, v);
    }
    const long at = (long)t * a.y_stride + tile * 16 + j;
    if (a.res) v += (float)static_cast<const T*>(a.res)[at];
    static_cast<T*>(a.y)[at] = (T)v;
  }
}

// y of more pairs: a token's parts from memory, eight at a time, and the residual.  A thread makes four channels.
template <typename T>
__global__ __launch_bounds__(256) void experts_add_kernel(const ExpertsArgs a) {
  const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4, t = (int)blockIdx.y;
  if (c >= a.channels) return;
  typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  const long at = (long)t * a.y_stride + c;
  four res = {};
  if (a.res) res = *reinterpret_cast<const four*>(static_cast<const T*>(a.res) + at);   // (on its way with the parts)
  floatx4 v = {0, 0, 0, 0};
  for (int s0 = 0; s0 < a.top_k; s0 += 8) {
    floatx4 part[8];
    int named[8];
    float weight[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int p = t * a.top_k + min(s0 + s, a.top_k - 1);
      named[s] = a.chosen[p];
      weight[s] = a.weights[p];
      part[s] = *reinterpret_cast<const floatx4*>(a.parts + (long)p * a.channels + c);
    }
#pragma unroll
    for (int s = 0; s < 8; ++s)   // (a pair that names no expert has no part: what stands in its place is not used)
      if (s0 + s < a.top_k && (unsigned)named[s] < (unsigned)a.experts)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(weight[s], part[s][j], v[j]);
  }
  four out;
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = (T)(a.res ? v[j] + (float)res[j] : v[j]);
  *reinterpret_cast<four*>(static_cast<T*>(a.y) + at) = out;
}

template <typename T, bool UP, int XL, int KS>
hipError_t launch_rows(const ExpertsArgs& a, const W4Layout& l, int n, hipStream_t st) {
  constexpr int W = 4, D = 2;
  const int units = (UP ? a.inter : a.channels) / 16, tiles = W / KS * (UP ? n : 2 * n), per_group = a.group_of(UP ? a.channels : a.inter) / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)((units + tiles - 1) / tiles), (unsigned)(a.by_pair ? a.pairs : a.experts)), block(W * 64);
  if (per_group % 4 == 0) hipLaunchKernelGGL((experts_rows_kernel<T, UP, XL, KS, D, W, 4>), grid, block, 0, st, a, l, fd, n);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((experts_rows_kernel<T, UP, XL, KS, D, W, 2>), grid, block, 0, st, a, l, fd, n);
  else hipLaunchKernelGGL((experts_rows_kernel<T, UP, XL, KS, D, W, 1>), grid, block, 0, st, a, l, fd, n);
  return hipGetLastError();
}

template <typename T, bool UP>
hipError_t launch_tiles(const ExpertsArgs& a, const W4Layout& l, hipStream_t st) {
  const int units = (UP ? a.inter : a.channels) / 16, tiles = UP ? 4 : 8, per_group = a.group_of(UP ? a.channels : a.inter) / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)((units + tiles - 1) / tiles), (unsigned)a.most_blocks), block(256);
  if (per_group % 4 == 0) hipLaunchKernelGGL((experts_tiles_kernel<T, UP, 4>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((experts_tiles_kernel<T, UP, 2>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((experts_tiles_kernel<T, UP, 1>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

template <typename T, int XL>
hipError_t launch_join(const ExpertsArgs& a, const W4Layout& l, hipStream_t st) {
  const int per_group = a.group_of(a.inter) / 32;
  const FastDiv fd = make_fastdiv((uint32_t)per_group);
  const dim3 grid((unsigned)(a.channels / 16)), block(kJoinWaves * 64);
  if (per_group % 4 == 0) hipLaunchKernelGGL((experts_join_kernel<T, XL, 4>), grid, block, 0, st, a, l, fd);
  else if (per_group % 2 == 0) hipLaunchKernelGGL((experts_join_kernel<T, XL, 2>), grid, block, 0, st, a, l, fd);
  else hipLaunchKernelGGL((experts_join_kernel<T, XL, 1>), grid, block, 0, st, a, l, fd);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const ExpertsArgs& a, hipStream_t st) {
  const W4Layout up = w4_layout(a.experts * 2 * a.inter, a.channels, a.group_of(a.channels), a.zeros != 0);
  const W4Layout down = w4_layout(a.experts * a.channels, a.inter, a.group_of(a.inter), a.zeros != 0);
  const long active = a.pairs < a.experts ? a.pairs : a.experts, up_waves = active * (a.inter / 16), down_waves = active * (a.channels / 32);
  const bool few = 4L * a.pairs <= a.experts, some = a.pairs <= 4L * a.experts;   // rows of an expert: one, seldom two; four on the mean
  // Tiles where an expert has six rows or more on the mean and enough tiles are there for the chip, or the rows are many.  us, rows of codes / tiles, 4, 8 and 16 rows: 2048 channels, 1408 beside
  // them, 32 experts, fp16 56 59 90 / 49 53 62, bf16 55 60 91 / 58 63 76, groups of 32 78 82 121 / 58 69 81; 4096, 1024, 64 experts, fp16 111 129 186 / 117 122 133, bf16 110 131 187 / 122 130 155,
  // 128 experts 215 262 381 / 217 241 275; 4096, 1024, 8 experts in groups of 64: 8 rows 34 / 48, 16 54 / 63, 32 96 / 100, 64 172 / 86.
  const long mean = a.pairs / a.experts;
  const bool tiled = mean > 32 || (mean >= 6 && (long)a.experts * ((a.inter + 63) / 64) >= 512);
  hipError_t e;
  if (tiled) {
    hipLaunchKernelGGL(experts_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
    if ((e = hipGetLastError())) return e;
  }
  if (!tiled && (few || some)) {
    if (few) e = up_waves >= 2048 ? launch_rows<T, true, 1, 2>(a, up, 1, st) : launch_rows<T, true, 1, 4>(a, up, 1, st);
    else e = up_waves >= 4096 ? launch_rows<T, true, 2, 1>(a, up, 1, st) : up_waves >= 2048 ? launch_rows<T, true, 2, 2>(a, up, 1, st) : launch_rows<T, true, 2, 4>(a, up, 1, st);
  } else {
    e = tiled ? launch_tiles<T, true>(a, up, st) : launch_rows<T, true, 4, 2>(a, up, 1, st);
  }
  if (e != hipSuccess) return e;
  // The join where its waves take one expert each, or two and there are workgroups enough to hide the second.  us of both launches, join / rows and their sum: 2048 channels, 4 pairs 13.8 / 17.2, 8 19.1 / 19.5,
  // 16 30.5 / 26.7, 32 44.8 / 35.6; 1024 channels, 8 pairs 20.9 / 21.0, 16 31.2 / 23.4; 4096 channels, 8 pairs 19.7 / 22.0, 16 28.2 / 30.2, 32 52.8 / 50.7; 7168 channels, 16 pairs 68 / 67, 48 137 / 132.
  if (a.pairs <= (a.channels >= 4096 ? kJoined : kJoinWaves)) return few ? launch_join<T, 1>(a, down, st) : some ? launch_join<T, 2>(a, down, st) : launch_join<T, 4>(a, down, st);
  if (!tiled && some) e = down_waves >= 4096 ? launch_rows<T, false, 2, 1>(a, down, down_waves >= 8192 ? 2 : 1, st) : launch_rows<T, false, 2, 2>(a, down, 1, st);
  else e = tiled ? launch_tiles<T, false>(a, down, st) : launch_rows<T, false, 4, 2>(a, down, 1, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((experts_add_kernel<T>), dim3((unsigned)((a.channels + 1023) / 1024), (unsigned)a.tokens), dim3(256), 0, st, a);
  return hipGetLastError();
}

constexpr int kPairs = 4096;   // of a launch at most
static_assert(kRouteTopK <= kPairs, "a token's pairs");
int tokens_at_once(const ExpertsArgs& a) { return kPairs / a.top_k; }
size_t blocks_of(int pairs, int experts) { return (size_t)(pairs < experts ? pairs : experts) + pairs / kBlock; }   // at most
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t experts_workspace_bytes(const ExpertsArgs& a) {
  const size_t pairs = (size_t)(a.tokens < tokens_at_once(a) ? a.tokens : tokens_at_once(a)) * a.top_k;
  return up256(pairs * a.inter * 2) + up256(pairs * a.channels * 4) + up256(pairs * 4) + up256(blocks_of((int)pairs, a.experts) * 12);
}

hipError_t launch_experts(const ExpertsArgs& args, int dtype, hipStream_t st) {
  const int most = tokens_at_once(args);
  for (long first = 0; first < args.tokens; first += most) {
    ExpertsArgs a = args;
    a.tokens = (int)(args.tokens - first < most ? args.tokens - first : most);
    a.pairs = a.tokens * a.top_k;
    a.by_pair = a.pairs <= a.experts;
    a.fd_top_k = make_fastdiv((uint32_t)a.top_k);
    const int64_t rows = first * 2;
    a.x = static_cast<const char*>(args.x) + rows * a.x_stride;
    a.y = static_cast<char*>(args.y) + rows * a.y_stride;
    if (a.res) a.res = static_cast<const char*>(args.res) + rows * a.y_stride;
    a.chosen = args.chosen + first * a.top_k;
    a.weights = args.weights + first * a.top_k;
    a.h = args.workspace;
    a.parts = reinterpret_cast<float*>(static_cast<char*>(args.workspace) + up256((size_t)a.pairs * a.inter * 2));
    a.sorted = reinterpret_cast<int*>(reinterpret_cast<char*>(a.parts) + up256((size_t)a.pairs * a.channels * 4));
    a.blocks = reinterpret_cast<int*>(reinterpret_cast<char*>(a.sorted) + up256((size_t)a.pairs * 4));
    a.most_blocks = (int)blocks_of(a.pairs, a.experts);
    if (hipError_t e = dtype == T_F16 ? launch_type<_Float16>(a, st) : launch_type<__bf16>(a, st)) return e;
  }
  return hipSuccess;
}

}  // namespace relay
