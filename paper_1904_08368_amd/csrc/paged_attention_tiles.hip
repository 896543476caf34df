// Attention of many query rows over a paged cache (prompts, long chunks): attn_tiles_kernel.
//
// 128 rows of a key head (a row is a token and one of the query heads that share the key head) to a workgroup, 32 to each of its four waves; 64 keys at a
// time, staged in LDS for all of them without passing through registers, two buffers, one barrier a tile.  Bound by the matrix cores and, close behind, by the
// exponentials and the LDS reads: a wave does 32 products of 32 x 32 x 16 on a tile (head_dim 128), 2048 exponentials in 32 instructions of quarter rate,
// and reads all 32 KB of it.  Two workgroups share a CU, so that one's softmax runs beside the other's products.
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

template <typename T, int DP, bool FULL>
__global__ __launch_bounds__(kTileWaves * 64, DP <= 128 ? 2 : 1) void attn_tiles_kernel(const AttnArgs a, const int groups, const int tiles) {
  typedef Mma<T> M;
  typedef typename M::vec vec;
    // keys of a tile; chunks of a row; steps of the two products; copies of a wave
  constexpr int KEYS = DP <= 128 ? 64 : 32, NB = KEYS / 32, CH = DP / 8, KS = DP / 16, DB = DP / 32, PER = KEYS * CH / (kTileWaves * 64);
  constexpr unsigned long long ALL = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
  __shared__ __attribute__((aligned(16))) T kv[2][2][KEYS * DP];    // [buffer][keys, values]
  __shared__ int s_odd, s_odd_at[kOddTiles];   // tiles whose values hold an infinity or a NaN, see below
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
  const int D = FULL ? DP : a.head_dim;
  // Key heads vary fastest, so that those of one XCD (a workgroup in eight) are the same few; the tiles with the most keys go first.
  const int grp = (int)blockIdx.x % groups, tile = tiles - 1 - (int)blockIdx.x / groups;
  const int b = grp / a.kv_heads, hk = grp - b * a.kv_heads;
  const Seq s(a, b);
  const int rows = min(s.nq, a.max_q_len) * a.group, r0 = tile * kTileRows;
  if (r0 >= rows) return;
  const unsigned flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f ? 0u : 0xffffffffu;
  const float c = keep ? fabsf(a.scale_log2) : 1.f;
  auto token_of = [&](int r) { return (int)fast_div((unsigned)min(r, rows - 1), a.fd_group); };
  // keys of the tile, of this wave's rows, and those that all of them see
  const int lo = s.first(a, token_of(r0)), hi = s.last(a, token_of(r0 + kTileRows - 1)) + 1;
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
  // Starts the copy of a tile; the keys that can be read.  The others' places are taken by the tile's first key that is read anyway.
  auto copy_tile = [&](int j0, int buf) {
    const int j = min(j0 + lane, hi - 1);
    const bool ok = lane < KEYS && j0 + lane < hi && (unsigned)pageno < (unsigned)a.num_pages;
    const int slot = j - (int)fast_div((unsigned)j, a.fd_page) * a.page_size;
    const long at = 2 * ((long)pageno * a.page_stride + (long)slot * a.slot_stride);
    const unsigned long long can = __ballot(ok);
    const long off = ok ? at : 0;
    const unsigned base = lds_address(&kv[buf][0][0]) + (unsigned)(wave * PER * 1024);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int place = (wave * PER + i) * 64 + lane, row = place / CH, p = place - row * CH;
      const long o = __shfl(off, row, 64);
      const int ck = k_chunk<CH>(row, p), cv = v_place<CH>(row, p);
      if (FULL || ck * 8 < D) lds_dma16_at(base + i * 1024, kbase + o + ck * 16);
      if (FULL || cv * 8 < D) lds_dma16_at(base + KEYS * DP * 2 + i * 1024, vbase + o + cv * 16);
    }
    return can;
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
  // rescaling, and probabilities of up to 256 are as exact as those of up to 1.
  float ref = kNegInf, l = 0.f;

  unsigned long long can = 0, can_next = 0;
  if (lo < hi) {
    look_up(lo);
    can_next = copy_tile(lo, 0);
    look_up(lo + KEYS);
  }
  int buf = 0;
  for (int j0 = lo; j0 < hi; j0 += KEYS, buf ^= 1) {
    // this tile's copies have arrived, those of all waves, and no wave reads the other buffer any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    can = can_next;
    if (j0 + KEYS < hi) {
      can_next = copy_tile(j0 + KEYS, buf ^ 1);
      look_up(j0 + 2 * KEYS);
    }
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
    if (j0 >= w_hi || j0 + KEYS <= w_lo) continue;
    const T* ks = kv[buf][0];
    const T* vs = kv[buf][1];
    floatx16 st[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) st[t][e] = 0.f;
      const int row = t * 32 + col;
#pragma unroll
      for (int k = 0; k < KS; ++k)
        st[t] = M::mfma32(*reinterpret_cast<const vec*>(ks + row * DP + k_place<CH>(row, 2 * k + h) * 8), qf[k], st[t]);
    }
    if (!whole) {
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int u = t * 32 + 8 * (e / 4) + 4 * h + e % 4, j = j0 + u;
          const bool seen = (can >> u & 1) && j >= my_first && j <= my_last;
          st[t][e] = seen ? st[t][e] : kNegInf;
        }
    }
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
    const float base = ref == kNegInf ? 0.f : ref;
    vec pf[2 * NB];
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) {
      uintx4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = pow2(fmaf(st[t / 2][8 * (t & 1) + 2 * e], c, -base)), p1 = pow2(fmaf(st[t / 2][8 * (t & 1) + 2 * e + 1], c, -base));
        sum += p0 + p1;
        w[e] = pack2<T>(p0, p1);
      }
      pf[t] = __builtin_bit_cast(vec, w);
    }
    l += sum;
    // values: this lane's piece of the rows 16 t + 4 h .. + 3 and of the rows 8 further on
    const int vrow = 4 * h + ((lane & 15) >> 2), vch = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), vhalf = (lane & 1) * 4;
    auto values = [&](int t, int d) {
      const int ra = 16 * t + vrow, rb = ra + 8;
      const uintx2 v0 = lds_transposed(vs + ra * DP + v_place<CH>(ra, d * 4 + vch) * 8 + vhalf);
      const uintx2 v1 = lds_transposed(vs + rb * DP + v_place<CH>(rb, d * 4 + vch) * 8 + vhalf);
      return (uintx4){v0[0], v0[1], v1[0], v1[1]};
    };
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] = M::mfma32(__builtin_bit_cast(vec, values(t, d)), pf[t], acc[d]);
  }
  l = sum_halves(l);

  // Values that were left out, tile by tile (a tile may stand in the list once for each wave: an infinity or a NaN added again is the same), or of all
  // tiles that are not whole if the list was too short.
  __syncthreads();
  const int found = __builtin_amdgcn_readfirstlane(s_odd);
  if (found) {
    const bool all = found > kOddTiles;
    for (int n = 0; n < (all ? (hi - lo + KEYS - 1) / KEYS : found); ++n) {
      const int j0 = all ? lo + n * KEYS : __builtin_amdgcn_readfirstlane(s_odd_at[n]);
      look_up(j0);
      const bool ok = lane < KEYS && j0 + lane < hi && (unsigned)pageno < (unsigned)a.num_pages;
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
  if (!row_ok) return;
  const bool none = my_last < my_first;
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

template <typename T, int DP>
hipError_t launch_dim(const AttnArgs& a, hipStream_t st) {
  const int groups = a.batch * a.kv_heads, tiles = (int)(((long)a.max_q_len * a.group + kTileRows - 1) / kTileRows);
  const dim3 grid((unsigned)(groups * tiles)), block(kTileWaves * 64);
  if (a.head_dim == DP) hipLaunchKernelGGL((attn_tiles_kernel<T, DP, true>), grid, block, 0, st, a, groups, tiles);
  else hipLaunchKernelGGL((attn_tiles_kernel<T, DP, false>), grid, block, 0, st, a, groups, tiles);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const AttnArgs& a, hipStream_t st) {
  const int d = a.head_dim;
  return d <= 64 ? launch_dim<T, 64>(a, st) : d <= 96 ? launch_dim<T, 96>(a, st) : d <= 128 ? launch_dim<T, 128>(a, st) : launch_dim<T, 256>(a, st);
}

}  // namespace

hipError_t launch_attention_tiles(const AttnArgs& a, int dtype, hipStream_t st) {
  return dtype == T_F16 ? launch_type<_Float16>(a, st) : launch_type<__bf16>(a, st);
}

}  // namespace relay
