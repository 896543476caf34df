// Attention of many query rows over a paged cache (prompts, long chunks): attn_tiles_kernel.
//
// 128 rows of a key head (a row is a token and one of the query heads that share the key head) to a workgroup, 32 to each of its four waves; 64 keys at a
// time, staged in LDS for all of them without passing through registers, two buffers, one barrier a step.  Bound by the matrix cores and, beside them, by vector
// instructions: on a step a wave does 32 products of 32 x 32 x 16 (head_dim 128) in 1024 clocks, and 2048 exponentials and what belongs to them in 990.  Two workgroups
// share a CU, so that one's softmax runs beside the other's products.  Where there are few tiles their keys are cut into parts, and a second
// kernel joins them.  Measured: 8192 tokens, 16 heads over 4 key heads, fp16, 293 to 303 us by box = 938 to 907 TFLOP/s; 512 tokens over 30000 keys, 32 over 8, 270 to 277 us; 64 tokens over
// them 55 us.  Other heads: 2 x 4096 tokens, 16 over 4 of 64, fp16, 96 us = 717 TFLOP/s; 4 x 2048 of 96, bf16, 56 us = 565; 2 x 2048 of 256, bf16, 124 us = 457 (one workgroup to a CU).
#include <algorithm>
#include <type_traits>

#include "attn_common.hpp"
#include "lds_dma.hpp"

namespace relay {
namespace {

constexpr int kTileRows = 128, kTileWaves = 4, kOddTiles = 16;

__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// Where chunk c (16 bytes) of a row lies within it: so that the 16 rows that read one chunk at a time, and the 8 rows by 4 chunks of a transposed
// read, fall on different banks.
template <int CH> __device__ __forceinline__ int k_place(int row, int c) {
  if constexpr (CH == 12) {
    const int t = c + ((row >> 2) & 3);
    return t >= 12 ? t - 12 : t;
  }
  return CH == 8 ? c ^ ((row >> 1) & 7) : c ^ (row & 15);
}
template <int CH> __device__ __forceinline__ int k_chunk(int row, int place) {
  if constexpr (CH == 12) {
    const int t = place - ((row >> 2) & 3);
    return t < 0 ? t + 12 : t;
  }
  return k_place<CH>(row, place);
}
template <int CH> __device__ __forceinline__ int v_place(int row, int c) {
  if constexpr (CH == 12) return c;   // (rows of 192 bytes: four rows already start on four different quarters of the banks)
  return CH == 8 ? c ^ (((row >> 1) & 1) << 2) : c ^ ((row & 3) << 2);
}

// How the work is cut: groups (a sequence's key head), tiles of rows of a group, parts of a tile's keys of `unit` steps each.
struct TilesPlan {
  int groups, tiles, parts, unit;
};

// The workgroups of a CU, by registers and LDS.
constexpr int workgroups_of_cu(int dp) { return dp <= 64 ? 3 : dp <= 128 ? 2 : 1; }
constexpr int tile_keys(int dp) { return dp <= 128 ? 64 : 32; }

// The keys of a tile of rows: steps of KEYS from `start` on, and into how many parts they are cut.
struct Span {
  int lo, hi, start, steps, parts;
  template <typename TokenOf>
  __device__ Span(const AttnArgs& a, const TilesPlan& pl, const Seq& s, int r0, int keys, int align, TokenOf token_of) {
    lo = s.first(a, token_of(r0));
    hi = s.last(a, token_of(r0 + kTileRows - 1)) + 1;
    start = lo & -align;
    steps = max(0, (hi - start + keys - 1) / keys);
    parts = max(1, min(pl.parts, (steps + pl.unit - 1) / pl.unit));
  }
  // first step of a part
  __device__ int first(int part) const { return (int)((long)steps * part / parts); }
};

// What a workgroup leaves of its part of a tile, in floats: the sums [d / 4][thread][4], then the reference and the sum of each row.
template <int DP> constexpr int cut_floats() { return kTileRows * DP + 2 * kTileRows; }

// FULL: head_dim is DP.  PAGED: the 16 keys that a wave copies of a step lie in one page.
template <typename T, int DP, bool FULL, bool PAGED>
__global__ __launch_bounds__(kTileWaves * 64, workgroups_of_cu(DP)) void attn_tiles_kernel(const AttnArgs a, const TilesPlan pl) {
  typedef Mma<T> M;
  typedef typename M::vec vec;
  // keys of a step; chunks of a row; steps of the two products; copies of a wave
  constexpr int KEYS = tile_keys(DP), NB = KEYS / 32, CH = DP / 8, KS = DP / 16, DB = DP / 32, PER = KEYS * CH / (kTileWaves * 64);
  constexpr unsigned long long ALL = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
  __shared__ __attribute__((aligned(16))) T kv[2][2][KEYS * DP];    // [buffer][keys, values]
  __shared__ int s_odd, s_odd_at[kOddTiles];   // tiles whose values hold an infinity or a NaN, see below
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
  const int D = FULL ? DP : a.head_dim;
  // Key heads vary fastest, so that those of one XCD (a workgroup in eight) are the same few; the tiles with the most keys go first.
  const int grp = (int)blockIdx.x % pl.groups, cut = (int)blockIdx.x / pl.groups, part = cut % pl.parts, tile = pl.tiles - 1 - cut / pl.parts;
  const int b = grp / a.kv_heads, hk = grp - b * a.kv_heads;
  const Seq s(a, b);
  const int rows = min(s.nq, a.max_q_len) * a.group, r0 = tile * kTileRows;
  if (r0 >= rows) return;
  auto token_of = [&](int r) { return (int)fast_div((unsigned)min(r, rows - 1), a.fd_group); };
  const Span span(a, pl, s, r0, KEYS, PAGED ? 16 : 1, token_of);
  if (part >= span.parts) return;
  const unsigned flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f ? 0u : 0xffffffffu;
  const float c = keep ? fabsf(a.scale_log2) : 1.f;
  // keys of this part, of this wave's rows, and those that all of them see
  const int hi = min(span.hi, span.start + span.first(part + 1) * KEYS), first = span.start + span.first(part) * KEYS, lo = max(span.lo, first);
  const int start = lo < hi ? first : hi;
  const int w0 = r0 + wave * 32, iw0 = token_of(w0), iw1 = token_of(w0 + 31);
  const int w_lo = s.first(a, iw0), w_hi = w0 < rows ? s.last(a, iw1) + 1 : 0;
  const int full_lo = s.first(a, token_of(r0 + kTileRows - 1)), full_hi = s.last(a, token_of(r0)) + 1;
  // this lane's row
  const int r = w0 + col, ri = token_of(r), token = s.start + ri, head = hk * a.group + min(r, rows - 1) - ri * a.group;
  const bool row_ok = r < rows && (unsigned)token < (unsigned)a.tokens;
  const int my_first = s.first(a, ri), my_last = s.last(a, ri);

  if (tid == 0) s_odd = 0;
  if constexpr (!FULL) {   // channels behind head_dim: zeros that no copy touches
    uintx4* z = reinterpret_cast<uintx4*>(&kv[0][0][0]);
    for (int i = tid; i < 4 * KEYS * CH; i += kTileWaves * 64) z[i] = (uintx4){0, 0, 0, 0};
    __syncthreads();
  }

  const int32_t* pages = a.page_table + (long)b * a.pages_per_seq;
  const char* kbase = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + (long)hk * a.head_stride);
  const char* vbase = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + (long)hk * a.head_stride);
  // Lane i looks up key i of a tile, a tile ahead of its copy.
  int pageno = 0;
  auto look_up = [&](int j0) {
    const int j = j0 + lane;
    pageno = pages[fast_div((unsigned)(j < hi ? j : lo), a.fd_page)];
  };
  // PAGED: where this lane's 16 bytes of each of the wave's copies lie, from the wave's first key on.
  unsigned k_at[PER], v_at[PER];
  if constexpr (PAGED)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int row = (i * 64 + lane) / CH, p = i * 64 + lane - row * CH, all = wave * (KEYS / 4) + row;
      k_at[i] = 2u * (unsigned)(row * (int)a.slot_stride) + 16u * (unsigned)k_chunk<CH>(all, p);
      v_at[i] = 2u * (unsigned)(row * (int)a.slot_stride) + 16u * (unsigned)v_place<CH>(all, p);
    }
  // The copies of a step: where they take from, and the keys that can be read.  In the others' places goes what can be read anyway: other keys of
  // the page, or of the cache's first.
  const char *kfrom = kbase, *vfrom = vbase;
  long from[PAGED ? 1 : PER];
  auto locate = [&](int j0) {
    const bool ok = (lane < KEYS) & (j0 + lane >= lo) & (j0 + lane < hi) & ((unsigned)pageno < (unsigned)a.num_pages);
    if constexpr (PAGED) {
      const int at = wave * (KEYS / 4), j = j0 + at, page = __builtin_amdgcn_readlane(pageno, at);
      const bool there = (j < hi) & ((unsigned)page < (unsigned)a.num_pages);
      const int slot = j - (int)fast_div((unsigned)j, a.fd_page) * a.page_size;
      const long off = 2 * ((long)(there ? page : 0) * a.page_stride + (long)(there ? slot : 0) * a.slot_stride);
      kfrom = kbase + off;
      vfrom = vbase + off;
    } else {
      const int j = min(j0 + lane, hi - 1);
      const int slot = j - (int)fast_div((unsigned)j, a.fd_page) * a.page_size;
      const long at = 2 * ((long)pageno * a.page_stride + (long)slot * a.slot_stride);
      const long off = ok ? at : 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) from[i] = __shfl(off, ((wave * PER + i) * 64 + lane) / CH, 64);
    }
    return __ballot(ok);
  };
  // one of the wave's copies of keys, of values
  auto copy_keys = [&](int buf, int i) {
    const int place = (wave * PER + i) * 64 + lane, row = place / CH, c = k_chunk<CH>(row, place - row * CH);
    const unsigned to = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(&kv[buf][0][0]) + (wave * PER + i) * 1024);
    if (FULL || c * 8 < D) {
      if constexpr (PAGED) lds_dma16_from(to, kfrom, k_at[i]);
      else lds_dma16_at(to, kbase + from[i] + c * 16);
    }
  };
  auto copy_values = [&](int buf, int i) {
    const int place = (wave * PER + i) * 64 + lane, row = place / CH, c = v_place<CH>(row, place - row * CH);
    const unsigned to = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(&kv[buf][1][0]) + (wave * PER + i) * 1024);
    if (FULL || c * 8 < D) {
      if constexpr (PAGED) lds_dma16_from(to, vfrom, v_at[i]);
      else lds_dma16_at(to, vbase + from[i] + c * 16);
    }
  };
  auto copy_all = [&](int buf) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      copy_keys(buf, i);
      copy_values(buf, i);
    }
  };

  vec qf[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    uintx4 t = {0, 0, 0, 0};
    if (row_ok && (FULL || k * 16 + h * 8 < D))
      t = *reinterpret_cast<const uintx4*>(static_cast<const T*>(a.q) + (long)token * a.q_token + (long)head * D + k * 16 + h * 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (t[e] & keep) ^ flip;
    qf[k] = __builtin_bit_cast(vec, t);
  }
  floatx16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
  // ref: what the exponents are taken relative to.  It follows the maximum only when that has outgrown it by 2^8: until then the sums need no
  // rescaling.  Probabilities are rounded to the tensor's type for the product with the values, as its operands are.  So the largest, which would be 1 and exact if
  // the reference were the maximum, is rounded too; l adds the rounded ones, so that what rounding does to a weight that is most of a row's it does
  // to both sides of the quotient.  Relative error with the unrounded ones in l / as it is / of the exact result rounded: 8192 tokens, fp16, 2.7e-4 / 2.5e-4 / 2.1e-4, chunks
  // over 9001 keys, bf16, 2.2e-3 / 2.1e-3 / 1.7e-3.  The additions stand between the second product's instructions: before them they took 3 % more time, there 0.3 %.
  float ref = kNegInf, l = 0.f;

  unsigned long long can = 0, can_next = 0;
  if (lo < hi) {
    look_up(start);
    can_next = locate(start);
    copy_all(0);
    look_up(start + KEYS);
  }
  int buf = 0, j0 = start;
  // One step; in between, the copies of the next one, spread out: issued together behind the barrier, a CU's 64 of them kept each wave waiting 930 of its 3800
  // clocks of a step.  MORE: there is a next one.
  auto step = [&](auto more) {
    constexpr bool MORE = decltype(more)::value;
    // this step's copies have arrived, those of all waves, and no wave reads the other buffer any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    can = can_next;
    auto next = [&]() {
      can_next = locate(j0 + KEYS);
      look_up(j0 + 2 * KEYS);
    };
    const bool whole = can == ALL && j0 >= full_lo && j0 + KEYS <= full_hi;   // (the same for all waves)
    if (!whole) {
      // Not all rows see all keys.  A product of zero and an infinity would be a NaN, also for the rows that do not see the key: such
      // values give way to zeros here, and go to the rows that see them one by one at the end.
      uintx4* v = reinterpret_cast<uintx4*>(kv[buf][1]);
      bool odd = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        uintx4 t = v[i * kTileWaves * 64 + tid];
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= not_finite<T>(t[e]);
        if (bad) {
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = only_finite<T>(t[e]);
          v[i * kTileWaves * 64 + tid] = t;
        }
        odd |= bad;
      }
      if (__ballot(odd) && lane == 0) {
        const int n = atomicAdd(&s_odd, 1);
        if (n < kOddTiles) s_odd_at[n] = j0;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    if (j0 >= w_hi || j0 + KEYS <= w_lo) {
      if constexpr (MORE) {
        next();
        copy_all(buf ^ 1);
      }
      return;
    }
    const T* ks = kv[buf][0];
    const T* vs = kv[buf][1];
    floatx16 st[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) st[t][e] = 0.f;
    // (product n: step n / NB of the reduction, keys 32 (n % NB) on; keys are read AHEAD products ahead)
    constexpr int N = NB * KS, AHEAD = 6;
    auto keys = [&](int n) {
      const int row = n % NB * 32 + col;
      return *reinterpret_cast<const vec*>(ks + row * DP + k_place<CH>(row, n / NB * 2 + h) * 8);
    };
    vec kf[AHEAD];
    __builtin_amdgcn_s_setprio(1);   // (products before the other workgroups' softmax: its waves fill the gaps by themselves)
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) kf[n] = keys(n);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      st[n % NB] = M::mfma32(kf[n % AHEAD], qf[n / NB], st[n % NB]);
      if (n + AHEAD < N) kf[n % AHEAD] = keys(n + AHEAD);
      if constexpr (MORE) {
        if (n == 1) next();
        if (n % (N / PER) == N / PER - 1) copy_keys(buf ^ 1, n / (N / PER));
      }
    }
    if (!whole) {
      // (counted from this lane's first key of the tile; the compiler would compute what depends on the lane ahead of the loop, and keep it in 100 registers)
      int h4 = 4 * h;
      asm volatile("" : "+v"(h4));
      const unsigned long long mine = can >> h4;
      const int from = my_first - j0 - h4, to = my_last - j0 - h4;
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int u = t * 32 + 8 * (e / 4) + e % 4;
          const bool seen = (mine >> u & 1) && u >= from && u <= to;
          st[t][e] = seen ? st[t][e] : kNegInf;
        }
    }
    __builtin_amdgcn_s_setprio(0);
    float bm = st[0][0];
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) bm = fmaxf(bm, st[t][e]);
    bm = max_halves(bm) * c;
    if (__ballot(bm > ref + 8.f)) {
      const float nr = bm > ref + 8.f ? bm : ref;
      const float alpha = ref == kNegInf ? 0.f : pow2(ref - nr);
      ref = nr;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] *= alpha;
    }
    const float base = ref == kNegInf ? 0.f : ref - M::kShiftTiles;
    vec pf[2 * NB];
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) {
      uintx4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = pow2(fmaf(st[t / 2][8 * (t & 1) + 2 * e], c, -base)), p1 = pow2(fmaf(st[t / 2][8 * (t & 1) + 2 * e + 1], c, -base));
        w[e] = pack2<T>(p0, p1);
      }
      pf[t] = __builtin_bit_cast(vec, w);
    }
    // values: this lane's piece of the rows 16 t + 4 h .. + 3 and of the rows 8 further on
    const int vrow = 4 * h + ((lane & 15) >> 2), vch = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), vhalf = (lane & 1) * 4;
    auto values = [&](int t, int d) {
      const int ra = 16 * t + vrow, rb = ra + 8;
      const uintx2 v0 = lds_transposed(vs + ra * DP + v_place<CH>(ra, d * 4 + vch) * 8 + vhalf);
      const uintx2 v1 = lds_transposed(vs + rb * DP + v_place<CH>(rb, d * 4 + vch) * 8 + vhalf);
      return (uintx4){v0[0], v0[1], v1[0], v1[1]};
    };
    constexpr int N2 = 2 * NB * DB, AHEAD2 = 4;
    uintx4 vf[AHEAD2];
#pragma unroll
    for (int n = 0; n < AHEAD2; ++n) vf[n] = values(n / DB, n % DB);
#pragma unroll
    for (int n = 0; n < N2; ++n) {
      acc[n % DB] = M::mfma32(__builtin_bit_cast(vec, vf[n % AHEAD2]), pf[n / DB], acc[n % DB]);
      if (n + AHEAD2 < N2) vf[n % AHEAD2] = values((n + AHEAD2) / DB, (n + AHEAD2) % DB);
#pragma unroll
      for (int e = n % DB * 4 / DB; e < (n % DB + 1) * 4 / DB; ++e) sum = M::add2(__builtin_bit_cast(uintx4, pf[n / DB])[e], sum);
      if constexpr (MORE)
        if (n % (N2 / PER) == 0) copy_values(buf ^ 1, n / (N2 / PER));
    }
    l += sum;
  };
  for (; j0 + KEYS < hi; j0 += KEYS, buf ^= 1) step(std::true_type());
  if (j0 < hi) step(std::false_type());
  l = sum_halves(l);

  // Values that were left out, tile by tile (a tile may stand in the list once for each wave: an infinity or a NaN added again is the same), or of all
  // tiles that are not whole if the list was too short.
  __syncthreads();
  const int found = __builtin_amdgcn_readfirstlane(s_odd);
  if (found) {
    const bool all = found > kOddTiles;
    for (int n = 0; n < (all ? (hi - start + KEYS - 1) / KEYS : found); ++n) {
      const int j0 = all ? start + n * KEYS : __builtin_amdgcn_readfirstlane(s_odd_at[n]);
      look_up(j0);
      const bool ok = lane < KEYS && j0 + lane >= lo && j0 + lane < hi && (unsigned)pageno < (unsigned)a.num_pages;
      const unsigned long long readable = __ballot(ok);
      if (all && readable == ALL && j0 >= full_lo && j0 + KEYS <= full_hi) continue;
#pragma unroll 1
      for (int u = 0; u < KEYS; ++u) {
        if (!(readable >> u & 1)) continue;
        const int j = j0 + u, slot = j - (int)fast_div((unsigned)j, a.fd_page) * a.page_size;
        const bool seen = j >= my_first && j <= my_last;
        const T* v = reinterpret_cast<const T*>(vbase) + (long)__shfl(pageno, u, 64) * a.page_stride + (long)slot * a.slot_stride;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int ch = d * 32 + 8 * (e / 4) + 4 * h + e % 4;
            const float x = FULL || ch < D ? (float)v[ch] : 0.f;
            acc[d][e] += seen && !(fabsf(x) < __builtin_inff()) ? x : 0.f;
          }
      }
    }
  }
  if (span.parts > 1) {
    float* const mine = static_cast<float*>(a.workspace) + kCounterBytes / 4 + ((size_t)(grp * pl.tiles + tile) * pl.parts + part) * cut_floats<DP>();
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<floatx4*>(mine + ((d * 4 + e / 4) * kTileWaves * 64 + tid) * 4) = (floatx4){acc[d][e], acc[d][e + 1], acc[d][e + 2], acc[d][e + 3]};
    if (h == 0) {
      mine[kTileRows * DP + 2 * (wave * 32 + col)] = ref;
      mine[kTileRows * DP + 2 * (wave * 32 + col) + 1] = l;
    }
    return;
  }
  if (!row_ok) return;
  const bool none = l == 0.f;   // no key that is seen and can be read
  const float inv = 1.f / l;
  T* const out = static_cast<T*>(a.out) + (long)token * a.out_token + (long)head * D;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int ch = d * 32 + 2 * e + 4 * h;
      uintx2 w = {pack2<T>(acc[d][e] * inv, acc[d][e + 1] * inv), pack2<T>(acc[d][e + 2] * inv, acc[d][e + 3] * inv)};
      if (none) w = (uintx2){0, 0};
      if (FULL || ch < D) *reinterpret_cast<uintx2*>(out + ch) = w;
    }
}

// Joins the parts of a tile, in their order; each thread the places of the same thread above, STEP of its float4s.
constexpr int kJoinStep = 2, kJoinBatch = 8;
template <typename T, int DP>
__global__ __launch_bounds__(kTileWaves * 64) void attn_join_kernel(const AttnArgs a, const TilesPlan pl, const int align) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5, col = lane & 31;
  const int grp = (int)blockIdx.x % pl.groups, tile = (int)blockIdx.x / pl.groups, b = grp / a.kv_heads, hk = grp - b * a.kv_heads;
  const Seq s(a, b);
  const int rows = min(s.nq, a.max_q_len) * a.group, r0 = tile * kTileRows;
  if (r0 >= rows) return;
  auto token_of = [&](int r) { return (int)fast_div((unsigned)min(r, rows - 1), a.fd_group); };
  const Span span(a, pl, s, r0, tile_keys(DP), align, token_of);
  if (span.parts == 1) return;
  const int r = r0 + wave * 32 + col, ri = token_of(r), token = s.start + ri, head = hk * a.group + min(r, rows - 1) - ri * a.group;
  const float* const parts = static_cast<const float*>(a.workspace) + kCounterBytes / 4 + (size_t)(grp * pl.tiles + tile) * pl.parts * cut_floats<DP>();
  const float* const stats = parts + kTileRows * DP + 2 * (wave * 32 + col);
  // (kJoinBatch parts at a time are on their way; those past the last are it again, and do not count)
  float m = kNegInf, l = 0.f;
  for (int u = 0; u < span.parts; u += kJoinBatch) {
    float mu[kJoinBatch];
#pragma unroll
    for (int e = 0; e < kJoinBatch; ++e) mu[e] = stats[(size_t)min(u + e, span.parts - 1) * cut_floats<DP>()];
#pragma unroll
    for (int e = 0; e < kJoinBatch; ++e) m = fmaxf(m, mu[e]);
  }
  floatx4 o[kJoinStep];
#pragma unroll
  for (int i = 0; i < kJoinStep; ++i) o[i] = (floatx4){0, 0, 0, 0};
  const int first = (int)blockIdx.y * kJoinStep;
  for (int u = 0; u < span.parts; u += kJoinBatch) {
    float mu[kJoinBatch], lu[kJoinBatch];
    floatx4 x[kJoinBatch][kJoinStep];
#pragma unroll
    for (int e = 0; e < kJoinBatch; ++e) {
      const size_t at = (size_t)min(u + e, span.parts - 1) * cut_floats<DP>();
      mu[e] = stats[at];
      lu[e] = stats[at + 1];
#pragma unroll
      for (int i = 0; i < kJoinStep; ++i) x[e][i] = *reinterpret_cast<const floatx4*>(parts + at + ((first + i) * kTileWaves * 64 + tid) * 4);
    }
#pragma unroll
    for (int e = 0; e < kJoinBatch; ++e)
      if (u + e < span.parts) {
        const float w = mu[e] == kNegInf ? 0.f : pow2(mu[e] - m);
        l += mu[e] == kNegInf ? lu[e] : lu[e] * w;   // (a part without a finite score brings zero, or a NaN)
#pragma unroll
        for (int i = 0; i < kJoinStep; ++i) o[i] += w * x[e][i];
      }
  }
  if (r >= rows || (unsigned)token >= (unsigned)a.tokens) return;
  const bool none = l == 0.f;
  const float inv = 1.f / l;
#pragma unroll
  for (int i = 0; i < kJoinStep; ++i) {
    const int ch = (first + i) * 8 + 4 * h;
    uintx2 w = {pack2<T>(o[i][0] * inv, o[i][1] * inv), pack2<T>(o[i][2] * inv, o[i][3] * inv)};
    if (none) w = (uintx2){0, 0};
    if (ch < a.head_dim) *reinterpret_cast<uintx2*>(static_cast<T*>(a.out) + (long)token * a.out_token + (long)head * a.head_dim + ch) = w;
  }
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }

// A part has 256 keys at least, and a tile 32 parts at most: beyond that the join costs more than the shorter parts save (us, at least 256 / 512 / 1024
// keys: 24 rows of 8 key heads over 4000 keys 17.6 / 20.4 / 29.8, over 30000 keys 50.9 / 50.8 / 44.2, which are 64 / 59 / 30 parts).
// All parts of a launch find room on the chip at once (as many, or half as many more: 512 tokens over 30000 keys 269 / 309, chunks of 509 tokens over 9001 45 / 47).
constexpr int kLeastKeys = 256, kMostParts = 32;

// (std::min and std::max: the unqualified ones take ints on the host, and a window may be up to 2^31 - 1)
TilesPlan tiles_plan(const AttnArgs& a, bool share) {
  const int dp = padded_dim(a.head_dim), keys = tile_keys(dp);
  TilesPlan p;
  p.groups = a.batch * a.kv_heads;
  p.tiles = (int)(((long)a.max_q_len * a.group + kTileRows - 1) / kTileRows);
  // steps of the longest tile
  const long tokens = std::min<long>(a.max_q_len, (long)kTileRows / a.group + 2), reach = a.causal && a.window > 0 ? a.window + tokens : a.max_kv_len;
  const long longest = std::max<long>(1, (std::min<long>(reach, a.max_kv_len) + keys - 1) / keys + 1);
  const long room = share ? std::max<long>(1, std::min<long>(kMostParts, 256L * workgroups_of_cu(dp) / std::max<long>(1, (long)p.groups * p.tiles))) : 1;
  p.unit = (int)std::max<long>(kLeastKeys / keys, (longest + room - 1) / room);
  p.parts = room > 1 ? (int)((longest + p.unit - 1) / p.unit) : 1;
  return p;
}

// 16 keys of a step lie in one page, and a lane's offset within them in 31 bits
bool one_page(const AttnArgs& a) { return a.page_size % 16 == 0 && a.slot_stride < 1 << 26; }

template <typename T, int DP, bool PAGED>
hipError_t launch_paged(const AttnArgs& a, hipStream_t st) {
  const TilesPlan p = tiles_plan(a, a.workspace != nullptr);
  const dim3 grid((unsigned)(p.groups * p.tiles * p.parts)), block(kTileWaves * 64);
  if (a.head_dim == DP) hipLaunchKernelGGL((attn_tiles_kernel<T, DP, true, PAGED>), grid, block, 0, st, a, p);
  else hipLaunchKernelGGL((attn_tiles_kernel<T, DP, false, PAGED>), grid, block, 0, st, a, p);
  if (p.parts > 1) {
    const dim3 join((unsigned)(p.groups * p.tiles), DP / 8 / kJoinStep);
    hipLaunchKernelGGL((attn_join_kernel<T, DP>), join, block, 0, st, a, p, PAGED ? 16 : 1);
  }
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_dim(const AttnArgs& a, hipStream_t st) {
  return one_page(a) ? launch_paged<T, DP, true>(a, st) : launch_paged<T, DP, false>(a, st);
}

template <typename T>
hipError_t launch_type(const AttnArgs& a, hipStream_t st) {
  const int d = a.head_dim;
  return d <= 64 ? launch_dim<T, 64>(a, st) : d <= 96 ? launch_dim<T, 96>(a, st) : d <= 128 ? launch_dim<T, 128>(a, st) : launch_dim<T, 256>(a, st);
}

}  // namespace

size_t attn_tiles_workspace_bytes(const AttnArgs& a) {
  const TilesPlan p = tiles_plan(a, true);
  if (p.parts == 1) return 0;
  const int dp = padded_dim(a.head_dim);
  return kCounterBytes + (size_t)p.groups * p.tiles * p.parts * (size_t)(kTileRows * dp + 2 * kTileRows) * 4;
}

hipError_t launch_attention_tiles(const AttnArgs& a, int dtype, hipStream_t st) {
  return dtype == T_F16 ? launch_type<_Float16>(a, st) : launch_type<__bf16>(a, st);
}

}  // namespace relay
