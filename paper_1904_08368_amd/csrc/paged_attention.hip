// Attention of new tokens over a paged cache:  o = sum_j softmax_j(scale q.k_j) v_j  over the keys a token sees.
//
// attn_rows_kernel: at most 16 query rows to a key head, one tile (a decode step, a few tokens at once).  A row is a token and one of the query heads
// that share the key head.  Bound by the bytes of the keys and values, which are read once.  A workgroup's waves take blocks
// of 32 keys in turn, each with a softmax of its own: keys go from memory straight into the A operands of S^T = K Q^T, values through a
// piece of LDS that only their wave uses, so that no wave waits for another before the end.
//
// Lengths differ from sequence to sequence and are known on the device only.  So the work is dealt out there: a tile's keys are units, the units
// of all tiles stand in one line, and each of as many workgroups as fit the chip at once takes an equal run of them.  Where there are fewer tiles than
// workgroups, a unit is made as long as lets every workgroup have one; else units are short and a run goes over several tiles.  A tile
// that lies within one run is finished by it; of others each workgroup leaves sums, maximum and weight in the workspace, and the one that arrives last
// joins them in the order of the line.
// Measured (key heads of 128 channels): 48 sequences of up to 8192 keys, 8 key heads, bf16, 212 us = 5.1 TB/s; one of 100001 keys, 4 key heads, fp16, 54 us, of which it streams
// 33 at 6 TB/s; one of 700 keys 11.9 us, of 200 8.7: an almost empty kernel is 2.4, the rest one trip to memory after another.
#include <algorithm>
#include <type_traits>

#include "attn_common.hpp"

namespace relay {
namespace {

constexpr int kRows = 16, kBlock = 32;
// workgroups that units are dealt out to, one to a CU, and so the most pieces of a tile; fewer of four waves where eight are the rule
constexpr int kMostPieces = 256;
constexpr int most_pieces(int dp, int waves) { return dp <= 128 && waves == 4 ? kMostPieces / 2 : kMostPieces; }

struct RowsPlan {
  int deal;        // 1: units of all tiles are dealt out over the grid; 0: a workgroup to a tile
  int unit;        // keys of a unit
};

// floats that a workgroup leaves behind: sums [16][DP], then the pair of maximum and sum of each row
template <int DP> constexpr int part_floats() { return kRows * DP + 2 * kRows; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What one sequence brings to the line of units: its tiles (one to a key head), and the keys that its rows see, which are the units of each.
struct Share {
  int tiles, lo, hi;
  __device__ Share(const AttnArgs& a, int b) : tiles(0), lo(0), hi(0) {
    if (b >= a.batch) return;
    const Seq s(a, b);
    const int nq = min(s.nq, a.max_q_len);
    if (nq <= 0) return;
    tiles = a.kv_heads;
    lo = s.first(a, 0);
    hi = s.last(a, nq - 1) + 1;
  }
  __device__ int units(int size) const { return max(1, (hi - lo + size - 1) / size); }
};

// How much the lanes up to this one have.
__device__ __forceinline__ int upto_lane(int n, int lane) {
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(n, o, 64);
    n += lane >= o ? t : 0;
  }
  return n;
}
// The line of units: the first 64 sequences' in the lanes, the others' read again where they are wanted.
struct Line {
  int size;             // keys of a unit
  int n, upto, total;   // units of sequence `lane`, of it and those ahead of it, of all
  __device__ Line() : size(0), n(0), upto(0), total(0) {}
  __device__ Line(const AttnArgs& a, int unit, int workers, int round, int lane) : size(unit) {
    const Share sh(a, lane);
    if (a.batch <= 64) {
      const int tiles = __builtin_amdgcn_readlane(upto_lane(sh.tiles, lane), 63);
      if (tiles <= workers) {
        // as long as needed for one to every worker: from an estimate, in a few steps (a unit to a tile is few enough)
        float keys = (float)sh.tiles * (float)(sh.hi - sh.lo);
        for (int o = 32; o > 0; o >>= 1) keys += __shfl_xor(keys, o, 64);
        size = max(round, uniform((int)fminf(keys / (float)workers, 1.0e9f)) + 63 & ~63);
        for (;;) {
          const int all = __builtin_amdgcn_readlane(upto_lane(sh.tiles * sh.units(size), lane), 63);
          if (all <= workers) break;
          size = (int)min((long)size * all / workers, 1L << 30) + 64 & ~63;
        }
      }
    }
    n = sh.tiles * sh.units(size);
    upto = upto_lane(n, lane);
    total = __builtin_amdgcn_readlane(upto, 63);
    for (int b0 = 64; b0 < a.batch; b0 += 64) {
      const Share next(a, b0 + lane);
      total += __builtin_amdgcn_readlane(upto_lane(next.tiles * next.units(size), lane), 63);
    }
  }
  // the sequence that a unit lies in, and the units ahead of that sequence
  __device__ void find(const AttnArgs& a, int unit, int lane, int& b, int& before) const {
    int nn = n, up = upto, ahead = 0;
    for (int b0 = 0;; b0 += 64) {
      const unsigned long long past = __ballot(unit < ahead + up);
      if (past || b0 + 64 >= a.batch) {
        const int at = past ? (int)__builtin_ctzll(past) : 63;
        b = b0 + at;
        before = ahead + __builtin_amdgcn_readlane(up - nn, at);
        return;
      }
      ahead += __builtin_amdgcn_readlane(up, 63);
      const Share next(a, b0 + 64 + lane);
      nn = next.tiles * next.units(size);
      up = upto_lane(nn, lane);
    }
  }
};

// Pieces go through the workspace in 8-byte stores and loads of device scope.  The XCDs' L2s are not coherent with each other, and to release or acquire
// ordinary ones would write back and invalidate a whole L2, under the feet of the workgroups that stream through it.
__device__ __forceinline__ void put_piece(float* p, float x, float y) {
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, (floatx2){x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uintx2 get_piece(const float* p) {
  return __builtin_bit_cast(uintx2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ floatx4 get_piece4(const float* p) {
  const uintx2 a = get_piece(p), b = get_piece(p + 2);
  return __builtin_bit_cast(floatx4, (uintx4){a[0], a[1], b[0], b[1]});
}

// FULL: head_dim is DP.  W: waves of a workgroup.
template <typename T, int DP, bool FULL, int W>
__global__ __launch_bounds__(W * 64, DP <= 128 ? 2 : 1) void attn_rows_kernel(const AttnArgs a, const RowsPlan pl) {
  typedef Mma<T> M;
  typedef typename M::vec vec;
  constexpr int KS = DP / 32, DT = DP / 16, PITCH = DP + 8, ROUND = W * kBlock;
  constexpr int SUMS = DP + 4;   // floats from one row's sums to the next in LDS: 16 rows on different banks
  static_assert(kBlock * PITCH * 2 >= kRows * SUMS * 4, "a wave's sums take the place of its values");
  __shared__ __attribute__((aligned(16))) T vs[W][kBlock * PITCH];
  __shared__ float sm[W][kRows], sl[W][kRows];
  __shared__ int s_last;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, col = lane & 15;
  const int D = FULL ? DP : a.head_dim;
  // (a negative scale: of -q, so that the largest score is the largest; a scale of zero: of zeros)
  const unsigned flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f ? 0u : 0xffffffffu;
  const float c = keep ? fabsf(a.scale_log2) : 1.f;
  T* const myv = vs[wave];

  // This workgroup's run of units.
  const int w_no = (int)blockIdx.x;
  int unit = 0, end = 1, run = 1, size = 0;
  int b = (int)blockIdx.y, before = 0, tiles = 1, units = 1, keys_lo = 0;   // the sequence at hand, units ahead of it, its tiles, their units, its first key
  int seq_end = 0;                                                          // the first unit behind it
  Line line;
  if (pl.deal) {
    line = Line(a, pl.unit, (int)gridDim.x, ROUND, lane);
    size = line.size;
    run = uniform(max(1, (line.total + (int)gridDim.x - 1) / (int)gridDim.x));
    unit = w_no * run;
    end = min(line.total, unit + run);
  }

  for (int piece = 0; unit < end; ++piece) {
    int hk, tile_unit = 0;   // key head; its first unit
    if (pl.deal && unit >= seq_end) line.find(a, unit, lane, b, before);
    const Seq s(a, b);
    if (!pl.deal || unit >= seq_end) {
      const Share sh(a, b);
      tiles = sh.tiles;
      keys_lo = sh.lo;
      if (pl.deal) {
        units = uniform(sh.units(size));
        seq_end = before + tiles * units;
      }
    }
    if (pl.deal) {
      hk = uniform((unit - before) / units);
      tile_unit = before + hk * units;
    } else {
      hk = (int)blockIdx.x;
      if (hk >= tiles) return;   // (no new tokens)
    }
    const int rows = min(s.nq, a.max_q_len) * a.group;
    const int stop = pl.deal ? min(end, tile_unit + units) : end;
    const bool whole_tile = !pl.deal || (unit == tile_unit && stop == tile_unit + units);
    const int i_max = min(s.nq, a.max_q_len) - 1;
    // the keys of this piece, as far as the tile's rows see them
    const int lo = max(s.first(a, 0), keys_lo + (unit - tile_unit) * size);
    const int hi = pl.deal ? min(s.last(a, i_max) + 1, keys_lo + (stop - tile_unit) * size) : s.last(a, i_max) + 1;
    // keys from full_lo to below full_hi are seen by all rows of the tile
    const int full_lo = s.first(a, i_max), full_hi = s.last(a, 0) + 1;
    // this lane's row
    const int r = col, ri = (int)fast_div((unsigned)min(r, rows - 1), a.fd_group);
    const int token = s.start + ri, head = hk * a.group + min(r, rows - 1) - ri * a.group;
    const bool row_ok = r < rows && (unsigned)token < (unsigned)a.tokens;
    const int my_first = s.first(a, ri), my_last = s.last(a, ri);

    const int32_t* pages = a.page_table + (long)b * a.pages_per_seq;
    const T* kbase = static_cast<const T*>(a.k) + (long)hk * a.head_stride + g * 8;
    const T* vbase = static_cast<const T*>(a.v) + (long)hk * a.head_stride + g * 8;

    // Page numbers of this lane's two keys (col and col + 16 of a block), asked for a block before their keys: a look-up on the way would
    // put a second trip through the caches into every block.
    int pageno[2];
    auto look_up = [&](int j0) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int j = j0 + t * 16 + col;
        pageno[t] = pages[fast_div((unsigned)(j < hi ? j : lo), a.fd_page)];
      }
    };
    // The keys' places in the cache, and which of the block's 32 keys can be read.
    long off[2] = {0, 0};
    unsigned can = 0;
    auto locate = [&](int j0) {
      unsigned long long m[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int j = j0 + t * 16 + col;
        const bool ok = j < hi && (unsigned)pageno[t] < (unsigned)a.num_pages;
        const int slot = j - (int)fast_div((unsigned)j, a.fd_page) * a.page_size;
        const long at = (long)pageno[t] * a.page_stride + (long)slot * a.slot_stride;
        off[t] = ok ? at : 0;
        m[t] = __ballot(ok);
      }
      can = ((unsigned)m[0] & 0xffffu) | ((unsigned)m[1] << 16);
    };
    uintx4 kf[2][KS], vf[2][KS];
    auto fetch = [&]() {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          if constexpr (!FULL) kf[t][k] = (uintx4){0, 0, 0, 0};
          if (FULL || k * 32 + g * 8 < D) kf[t][k] = *reinterpret_cast<const uintx4*>(kbase + off[t] + k * 32);
        }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          if constexpr (!FULL) vf[t][k] = (uintx4){0, 0, 0, 0};
          if (FULL || k * 32 + g * 8 < D) vf[t][k] = *reinterpret_cast<const uintx4*>(vbase + off[t] + k * 32);
        }
    };

    int j0 = lo + wave * kBlock;
    if (j0 < hi) {
      look_up(j0);
      locate(j0);
      fetch();
      look_up(j0 + ROUND);
    }
    vec qf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uintx4 t = {0, 0, 0, 0};
      if (row_ok && (FULL || k * 32 + g * 8 < D))
        t = *reinterpret_cast<const uintx4*>(static_cast<const T*>(a.q) + (long)token * a.q_token + (long)head * D + k * 32 + g * 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = (t[e] & keep) ^ flip;
      qf[k] = __builtin_bit_cast(vec, t);
    }
    floatx4 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = (floatx4){0, 0, 0, 0};
    float m = kNegInf, l = 0.f;
    // One block: scores, softmax, output; in between the next block's keys and values are asked for.  MORE: there is a next one.  (As a
    // condition inside the loop it would have the compiler keep two sets of them.)
    auto block = [&](auto more) {
      constexpr bool MORE = decltype(more)::value;
      floatx4 st[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        st[t] = (floatx4){0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) st[t] = M::mfma16(__builtin_bit_cast(vec, kf[t][k]), qf[k], st[t]);
      }
      const unsigned readable = can;
      unsigned long long odd = 0;   // keys with an infinity or a NaN among their values (bits 0..15, 32..47: first and second 16)
      const bool shared = j0 < full_lo || min(j0 + kBlock, hi) > full_hi;   // some of the rows may not see all of its keys
      if (shared || readable != 0xffffffffu) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bool ok = readable >> (t * 16 + col) & 1;
          bool bad = false;
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned v = vf[t][k][e];
              vf[t][k][e] = ok ? v : 0u;
              if (shared) bad |= ok && not_finite<T>(v);
            }
          if (shared) {
            unsigned long long bl = __ballot(bad);
            bl |= bl >> 32;
            odd |= ((bl | bl >> 16) & 0xffffull) << (32 * t);
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int u = t * 16 + g * 4 + e, j = j0 + u;
            const bool seen = (readable >> u & 1) && j >= my_first && j <= my_last;
            st[t][e] = seen ? st[t][e] : kNegInf;
          }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < KS; ++k) *reinterpret_cast<uintx4*>(myv + (t * 16 + col) * PITCH + k * 32 + g * 8) = vf[t][k];
      if constexpr (MORE) {
        locate(j0 + ROUND);
        fetch();
        look_up(j0 + 2 * ROUND);
      }
      float bm = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
      bm = max_quarters(bm);
      const float mn = fmaxf(m, bm), base = mn == kNegInf ? 0.f : mn * c;
      const float alpha = pow2(fmaf(m, c, -base));
      m = mn;
      float sum = 0.f;
      uintx4 pw;
      // Rounded to the tensor's type for the product with the values, as its operands are.  The largest of each block so far is a power of two and loses nothing;
      // the others' rounding adds up to less than the result's own (relative error of 48 sequences, bf16, 1.7e-3, as of the exact result rounded).
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          st[t][e] = pow2(fmaf(st[t][e], c, M::kShiftRows - base));
          sum += st[t][e];
        }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        pw[2 * t] = pack2<T>(st[t][0], st[t][1]);
        pw[2 * t + 1] = pack2<T>(st[t][2], st[t][3]);
      }
      l = fmaf(l, alpha, sum);
      const vec pf = __builtin_bit_cast(vec, pw);
      const T* at = myv + (g * 4 + (col >> 2)) * PITCH + (col & 3) * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        acc[d] *= alpha;
        const uintx2 v0 = lds_transposed(at + d * 16), v1 = lds_transposed(at + d * 16 + 16 * PITCH);
        uintx4 v = {v0[0], v0[1], v1[0], v1[1]};
        // A product of zero and an infinity would be a NaN, also for the rows that do not see the key: such values are left
        // out of the matrix product and go to the rows that see them one by one.
        if (odd)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = only_finite<T>(v[e]);
        acc[d] = M::mfma16(__builtin_bit_cast(vec, v), pf, acc[d]);
      }
      if (odd) {
        for (int u = 0; u < kBlock; ++u) {
          if (!(odd >> (u + (u & 16)) & 1)) continue;
          const bool seen = (readable >> u & 1) && j0 + u >= my_first && j0 + u <= my_last;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = (float)myv[u * PITCH + d * 16 + g * 4 + e];
              acc[d][e] += seen && !(fabsf(v) < __builtin_inff()) ? v : 0.f;
            }
        }
      }
    };
    for (; j0 + ROUND < hi; j0 += ROUND) block(std::true_type());
    if (j0 < hi) block(std::false_type());
    l = sum_quarters(l);

    // The waves' results, on the scale of the largest maximum.  (From here on by a copy of the thread's number that the compiler has to take
    // as new in every piece: it would compute the addresses below ahead of all pieces and keep them in 60 registers.)
    int tid_c = tid;
    asm volatile("" : "+v"(tid_c));
    const int col_c = tid_c & 15, g_c = (tid_c & 63) >> 4;
    if (g_c == 0) {
      sm[wave][col_c] = m;
      sl[wave][col_c] = l;
    }
    __syncthreads();
    float mt = kNegInf;
#pragma unroll
    for (int w = 0; w < W; ++w) mt = fmaxf(mt, sm[w][col_c]);
    const float own = m == kNegInf ? 0.f : pow2((m - mt) * c);
    float* const part = reinterpret_cast<float*>(vs[wave]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      if (col_c < rows) *reinterpret_cast<floatx4*>(part + col_c * SUMS + d * 16 + g_c * 4) = m == kNegInf ? (floatx4){0, 0, 0, 0} : acc[d] * own;
    __syncthreads();
    float* const slots = pl.deal ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + kCounterBytes) : nullptr;
    float* const mine = pl.deal ? slots + (size_t)(2 * w_no + (piece > 0 ? 1 : 0)) * part_floats<DP>() : nullptr;

    // one float4 of the output; row `cc` of the tile
    auto put = [&](int cc, int d, floatx4 o, float lt) {
      const int ii = (int)fast_div((unsigned)cc, a.fd_group);
      const int tk = s.start + ii;
      if ((unsigned)tk >= (unsigned)a.tokens) return;
      const float inv = 1.f / lt;
      uintx2 w = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
      if (lt == 0.f) w = (uintx2){0, 0};   // (no key that is seen and can be read)
      *reinterpret_cast<uintx2*>(static_cast<T*>(a.out) + (long)tk * a.out_token + (long)(hk * a.group + cc - ii * a.group) * D + d) = w;
    };
    for (int it = tid_c; it < rows * (DP / 4); it += W * 64) {
      const int cc = it / (DP / 4), d = it % (DP / 4) * 4;
      if (!FULL && d >= D) continue;
      floatx4 o = {0, 0, 0, 0};
      float mm = kNegInf, lt = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        o += *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(vs[w]) + cc * SUMS + d);
        mm = fmaxf(mm, sm[w][cc]);
      }
#pragma unroll
      for (int w = 0; w < W; ++w) lt += sm[w][cc] == kNegInf ? sl[w][cc] : sl[w][cc] * pow2((sm[w][cc] - mm) * c);
      if (whole_tile) {
        put(cc, d, o, lt);
        continue;
      }
      put_piece(mine + cc * DP + d, o[0], o[1]);
      put_piece(mine + cc * DP + d + 2, o[2], o[3]);
      if (d == 0) put_piece(mine + kRows * DP + 2 * cc, mm, lt);
    }
    unit = stop;
    if (whole_tile) {
      if (!pl.deal) return;
      __syncthreads();   // (the next piece takes the waves' LDS)
      continue;
    }

    // The workgroup that counts itself last, behind every wave's stores, joins the tile.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int w_first = uniform(tile_unit / run), w_last = uniform((tile_unit + units - 1) / run);
    const int pieces = w_last - w_first + 1;
    if (tid == 0) {
      unsigned* cnt = static_cast<unsigned*>(a.workspace) + (b * a.kv_heads + hk) * 16;
      const unsigned old = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = old == (unsigned)(pieces - 1);
      if (s_last) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) continue;
    // the first of them may have come to this tile behind another one, the others start with it
    auto slot = [&](int u) { return slots + (size_t)(2 * (w_first + u) + (u == 0 && w_first * run < tile_unit ? 1 : 0)) * part_floats<DP>(); };
    // Where the rows' float4s are fewer than the threads, several threads share one: thread group `sub` of `subs` takes every subs-th piece.  The first
    // JB of a thread's loads (each a trip to memory: other XCDs wrote the pieces) are on their way while the weights are made.
    constexpr int THREADS = W * 64, JB = 8, PIECES = most_pieces(DP, W);
    const int items = rows * (DP / 4), subs = max(1, THREADS / items), sub = subs > 1 ? tid_c / items : 0;
    auto fetch_pieces = [&](int it, int u, floatx4 (&t)[JB]) {
#pragma unroll
      for (int e = 0; e < JB; ++e) t[e] = get_piece4(slot(min(u + e * subs, pieces - 1)) + it / (DP / 4) * DP + it % (DP / 4) * 4);
    };
    auto wanted = [&](int it) { return it < items && sub < subs && (FULL || it % (DP / 4) * 4 < D); };
    floatx4 t[JB];
    if (wanted(tid_c - sub * items)) fetch_pieces(tid_c - sub * items, sub, t);
    // maxima [piece][16] and sums [piece][16]; each wave makes weights of some rows' maxima, then all threads add up the pieces
    float* const weight = reinterpret_cast<float*>(vs[0]);
    float* const lsum = weight + PIECES * kRows;
    static_assert(sizeof(vs) >= (2 * PIECES + 1) * kRows * 4 && PIECES * kRows * 4 >= THREADS * 16, "LDS of the join");
    float* const row_sum = lsum + PIECES * kRows;
#pragma unroll 2
    for (int i = tid_c; i < pieces * kRows; i += THREADS)
      if (i % kRows < rows) {
        const uintx2 p = get_piece(slot(i / kRows) + kRows * DP + 2 * (i % kRows));
        weight[i] = __builtin_bit_cast(float, (unsigned)p[0]);
        lsum[i] = __builtin_bit_cast(float, (unsigned)p[1]);
      }
    __syncthreads();
    for (int cc = wave; cc < rows; cc += W) {
      float mm = kNegInf, lt = 0.f;
      for (int u = lane; u < pieces; u += 64) mm = fmaxf(mm, weight[u * kRows + cc]);
      for (int o = 32; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o, 64));
      for (int u = lane; u < pieces; u += 64) {
        const float mu = weight[u * kRows + cc], w = mu == kNegInf ? 0.f : pow2((mu - mm) * c);
        lt += mu == kNegInf ? lsum[u * kRows + cc] : lsum[u * kRows + cc] * w;
        weight[u * kRows + cc] = w;
      }
      for (int o = 32; o > 0; o >>= 1) lt += __shfl_xor(lt, o, 64);
      if (lane == 0) row_sum[cc] = lt;
    }
    __syncthreads();
    floatx4* const shared_sums = reinterpret_cast<floatx4*>(lsum);
    for (int it0 = 0; it0 < items; it0 += THREADS) {
      const int it = it0 + tid_c - sub * items, cc = it / (DP / 4);
      floatx4 o = {0, 0, 0, 0};
      if (wanted(it))
        for (int u = sub; u < pieces; u += JB * subs) {
          if (it0 > 0 || u > sub) fetch_pieces(it, u, t);
#pragma unroll
          for (int e = 0; e < JB; ++e) o += u + e * subs < pieces ? t[e] * weight[(u + e * subs) * kRows + cc] : (floatx4){0, 0, 0, 0};
        }
      if (subs > 1) {
        shared_sums[tid_c] = o;
        __syncthreads();
        if (sub == 0)
          for (int e = 1; e < subs; ++e) o += shared_sums[e * items + it];
      }
      if (wanted(it) && sub == 0) put(cc, it % (DP / 4) * 4, o, row_sum[cc]);
    }
    __syncthreads();
  }
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }

struct RowsGrid {
  RowsPlan plan;
  dim3 grid;
  int waves;
};

// (std::min: the unqualified one takes ints on the host, and a window may be up to 2^31 - 1)
RowsGrid rows_plan(const AttnArgs& a, bool share) {
  RowsGrid p;
  const int dp = padded_dim(a.head_dim);
  const long tiles = (long)a.batch * a.kv_heads;
  // the most keys between the first and the last that a sequence's rows see
  const long keys = a.window > 0 && a.causal ? std::min<long>(a.max_kv_len, (long)a.window + a.max_q_len) : a.max_kv_len;
  // Keys are shared out where there are more than eight waves take at once, unless there are tiles for three workgroups out of four and no sequence is long: then
  // finding the shares and joining costs more than it evens out (us, shared out / a workgroup to a tile: one sequence of 200 keys, 8 key heads 11.6 / 8.6;
  // 24 of up to 1500 33.2 / 28.7, 16 of them 22.9 / 27.5; 200 of up to 900, 4 key heads 72 / 55, 128 of up to 4000 131 / 146).
  p.plan.deal = share && tiles <= kCounters && keys > 8 * kBlock && (tiles < kMostPieces * 3 / 4 || keys > 64 * kBlock);
  // Eight waves where their registers leave a CU room for them.  Four where rounds of theirs do not even give half of the CUs one: less to launch
  // and to join (us, four / eight waves: one sequence of 700 keys, 8 key heads 11.8 / 14.5, 1500 keys 12.0 / 14.8; 8 sequences of 3000 keys 35.9 / 23.4).
  // Four, too, where every CU gets two tiles or more: one's end runs beside the other's stream (200 sequences of up to 900 keys, 4 key heads 54.5 / 58.6).
  const bool four = p.plan.deal ? tiles * ((keys + 4 * kBlock - 1) / (4 * kBlock)) <= most_pieces(dp, 4) : tiles >= 2 * kMostPieces;
  p.waves = dp > 128 || four ? 4 : 8;
  const int round = p.waves * kBlock;
  // A unit is a round of the waves; where there are more of those than workgroups, a quarter of one, so that their shares come out more even
  // (48 sequences of up to 8192 keys, 8 key heads: 211 us, of whole rounds 213; 100 of up to 2000, 2 key heads 40.1 and 41.3).
  p.plan.unit = tiles * ((keys + round - 1) / round) > kMostPieces ? round / 4 : round;
  const long units = (keys + p.plan.unit - 1) / p.plan.unit;
  if (tiles * units >= 1L << 30) p.plan.deal = 0;
  if (p.plan.deal) p.grid = dim3((unsigned)std::min<long>(tiles * units, most_pieces(dp, p.waves)));
  else p.grid = dim3((unsigned)a.kv_heads, (unsigned)a.batch);
  return p;
}

template <typename T, int DP, int W>
hipError_t launch_waves(const AttnArgs& a, const RowsGrid& p, hipStream_t st) {
  if (a.head_dim == DP) hipLaunchKernelGGL((attn_rows_kernel<T, DP, true, W>), p.grid, dim3(W * 64), 0, st, a, p.plan);
  else hipLaunchKernelGGL((attn_rows_kernel<T, DP, false, W>), p.grid, dim3(W * 64), 0, st, a, p.plan);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_dim(const AttnArgs& a, const RowsGrid& p, hipStream_t st) {
  return p.waves == 4 ? launch_waves<T, DP, 4>(a, p, st) : launch_waves<T, DP, 8>(a, p, st);
}

template <typename T>
hipError_t launch_rows(const AttnArgs& a, hipStream_t st) {
  const RowsGrid p = rows_plan(a, a.workspace != nullptr);
  switch (padded_dim(a.head_dim)) {
    case 64: return launch_dim<T, 64>(a, p, st);
    case 96: return launch_dim<T, 96>(a, p, st);
    case 128: return launch_dim<T, 128>(a, p, st);
    default: return launch_waves<T, 256, 4>(a, p, st);
  }
}

}  // namespace

// More rows than one tile go to the other kernel, whose tiles read the keys once for 128 (us, this kernel with a tile more for every 16 rows / the other: 24 rows
// of 8 key heads, one sequence of 4000 keys 18.6 / 17.6, of 30000 44.9 / 44.2, 8 sequences of 30000 234 / 171; 96 rows, one of 30000 108 / 44).
static bool many_rows(const AttnArgs& a) { return (long)a.max_q_len * a.group > kRows; }

size_t attn_workspace_bytes(const AttnArgs& a) {
  if (a.max_q_len == 0) return 0;
  if (many_rows(a)) return attn_tiles_workspace_bytes(a);
  const RowsGrid p = rows_plan(a, true);
  if (!p.plan.deal) return 0;
  return kCounterBytes + (size_t)p.grid.x * 2 * (size_t)(kRows * padded_dim(a.head_dim) + 2 * kRows) * 4;
}

bool attn_fits(const AttnArgs& a) {
  return a.kv_heads < 65536 && a.batch < 65536 && a.max_kv_len <= 1 << 30 && (double)a.max_q_len * a.group * a.kv_heads < 1073741824.0 &&
         (double)a.batch * a.kv_heads * ((double)a.max_q_len * a.group / 128 + 1) < 8388608.0;   // (workgroups of the larger tiles)
}

hipError_t launch_attention(const AttnArgs& a, int dtype, hipStream_t st) {
  if (many_rows(a)) return launch_attention_tiles(a, dtype, st);
  return dtype == T_F16 ? launch_rows<_Float16>(a, st) : launch_rows<__bf16>(a, st);
}

}  // namespace relay
