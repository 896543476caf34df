// Attention of new tokens over a paged cache:  o = sum_j softmax_j(scale q.k_j) v_j  over the keys a token sees.
//
// attn_rows_kernel: few query rows to a key head (a decode step, a short chunk).  A row is a token and one of the query heads that share the key
// head, 16 rows to a workgroup: bound by the bytes of the keys and values, which every workgroup reads once for its 16 rows.  The workgroup's four
// waves take blocks of 32 keys in turn, each with a softmax of its own: keys go from memory straight into the A operands of S^T = K Q^T,
// values through a piece of LDS that only their wave uses, so that no wave waits for another before the end.  Where there are few workgroups,
// a sequence's keys are shared out in chunks; partial results meet in the workspace.
#include "attn_common.hpp"

namespace relay {
namespace {

constexpr int kRows = 16, kBlock = 32, kWaves = 4;
// Arrival counters lie 64 bytes apart in front of the workspace, in a region of their own that is the same for every call.
constexpr int kCounters = 1024;
constexpr size_t kCounterBytes = (size_t)kCounters * 64;

struct RowsPlan {
  int row_tiles, chunks, chunk;   // tiles of 16 rows of a sequence; chunks of `chunk` keys
};

// floats that a workgroup leaves behind: sums [16][DP], then maximum and sum of each row
template <int DP> constexpr int part_floats() { return kRows * DP + 2 * kRows; }

template <typename T, int DP>
__global__ __launch_bounds__(kWaves * 64) void attn_rows_kernel(const AttnArgs a, const RowsPlan pl) {
  typedef Mma<T> M;
  typedef typename M::vec vec;
  constexpr int KS = DP / 32, DT = DP / 16, PITCH = DP + 8;
  static_assert(kBlock * PITCH * 2 >= kRows * DP * 4, "a wave's sums take the place of its values");
  __shared__ __attribute__((aligned(16))) T vs[kWaves][kBlock * PITCH];
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  __shared__ int s_last;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, col = lane & 15;
  const int chunk_no = (int)blockIdx.x / pl.row_tiles, tile = (int)blockIdx.x - chunk_no * pl.row_tiles;
  const int hk = (int)blockIdx.y, b = (int)blockIdx.z;
  const Seq s(a, b);
  const int rows = min(s.nq, a.max_q_len) * a.group, r0 = tile * kRows;
  if (r0 >= rows) return;
  const int i_min = (int)fast_div((unsigned)r0, a.fd_group), i_max = (int)fast_div((unsigned)min(r0 + kRows - 1, rows - 1), a.fd_group);
  const int lo = s.first(a, i_min), hi = s.last(a, i_max) + 1;
  const int active = pl.chunks == 1 ? 1 : max(1, (hi - lo + pl.chunk - 1) / pl.chunk);
  if (chunk_no >= active) return;
  const int c_lo = lo + chunk_no * pl.chunk, c_hi = min(hi, c_lo + pl.chunk);
  // keys from full_lo to below full_hi are seen by all rows of the tile
  const int full_lo = s.first(a, i_max), full_hi = s.last(a, i_min) + 1;
  // this lane's row
  const int r = r0 + col, ri = (int)fast_div((unsigned)min(r, rows - 1), a.fd_group);
  const int token = s.start + ri, head = hk * a.group + min(r, rows - 1) - ri * a.group;
  const bool row_ok = r < rows && (unsigned)token < (unsigned)a.tokens;
  const int my_first = s.first(a, ri), my_last = s.last(a, ri);
  const int D = a.head_dim;

  vec qf[KS];
  // (a negative scale: of -q, so that the largest score is the largest; a scale of zero: of zeros)
  const unsigned flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f ? 0u : 0xffffffffu;
  const float c = keep ? fabsf(a.scale_log2) : 1.f;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    uintx4 t = {0, 0, 0, 0};
    if (row_ok && k * 32 + g * 8 < D)
      t = *reinterpret_cast<const uintx4*>(static_cast<const T*>(a.q) + (long)token * a.q_token + (long)head * D + k * 32 + g * 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (t[e] & keep) ^ flip;
    qf[k] = __builtin_bit_cast(vec, t);
  }
  const int32_t* pages = a.page_table + (long)b * a.pages_per_seq;
  const T* kbase = static_cast<const T*>(a.k) + (long)hk * a.head_stride + g * 8;
  const T* vbase = static_cast<const T*>(a.v) + (long)hk * a.head_stride + g * 8;

  // The place of this lane's two keys (col and col + 16 of a block) in the cache, and which of the block's 32 keys can be read.
  long off[2] = {0, 0};
  unsigned can = 0;
  auto locate = [&](int j0) {
    unsigned long long m[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = j0 + t * 16 + col;
      const bool in = j < c_hi;
      const int jj = in ? j : c_lo;
      const unsigned pg = fast_div((unsigned)jj, a.fd_page);
      const int page = pages[pg];
      const bool ok = in && (unsigned)page < (unsigned)a.num_pages;
      off[t] = ok ? (long)page * a.page_stride + (long)(jj - (int)pg * a.page_size) * a.slot_stride : 0;
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
        kf[t][k] = (uintx4){0, 0, 0, 0};
        if (DP == D || k * 32 + g * 8 < D) kf[t][k] = *reinterpret_cast<const uintx4*>(kbase + off[t] + k * 32);
      }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        vf[t][k] = (uintx4){0, 0, 0, 0};
        if (DP == D || k * 32 + g * 8 < D) vf[t][k] = *reinterpret_cast<const uintx4*>(vbase + off[t] + k * 32);
      }
  };

  floatx4 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = (floatx4){0, 0, 0, 0};
  float m = kNegInf, l = 0.f;
  T* const myv = vs[wave];
  int j0 = c_lo + wave * kBlock;
  if (j0 < c_hi) {
    locate(j0);
    fetch();
  }
  for (; j0 < c_hi; j0 += kWaves * kBlock) {
    floatx4 st[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      st[t] = (floatx4){0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k) st[t] = M::mfma16(__builtin_bit_cast(vec, kf[t][k]), qf[k], st[t]);
    }
    const unsigned readable = can;
    const bool whole = readable == 0xffffffffu && j0 >= full_lo && j0 + kBlock <= full_hi;   // (uniform)
    unsigned long long odd = 0;   // keys with an infinity or a NaN among their values (bits 0..15, 32..47: first and second 16)
    if (!whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool ok = readable >> (t * 16 + col) & 1;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vf[t][k][e] = ok ? vf[t][k][e] : 0u;
            bad |= not_finite<T>(vf[t][k][e]);
          }
        unsigned long long bl = __ballot(bad);
        bl |= bl >> 32;
        odd |= ((bl | bl >> 16) & 0xffffull) << (32 * t);
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
    if (j0 + kWaves * kBlock < c_hi) {
      locate(j0 + kWaves * kBlock);
      fetch();
    }
    float bm = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
    bm = max_quarters(bm);
    const float mn = fmaxf(m, bm), base = mn == kNegInf ? 0.f : mn * c;
    const float alpha = pow2(fmaf(m, c, -base));
    m = mn;
    float sum = 0.f;
    uintx4 pw;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        st[t][e] = pow2(fmaf(st[t][e], c, -base));
        sum += st[t][e];
      }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      pw[2 * t] = pack2<T>(st[t][0], st[t][1]);
      pw[2 * t + 1] = pack2<T>(st[t][2], st[t][3]);
    }
    l = fmaf(l, alpha, sum);
    const vec pf = __builtin_bit_cast(vec, pw);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      acc[d] *= alpha;
      const T* at = myv + (g * 4 + (col >> 2)) * PITCH + d * 16 + (col & 3) * 4;
      const uintx2 v0 = lds_transposed(at), v1 = lds_transposed(at + 16 * PITCH);
      uintx4 v = {v0[0], v0[1], v1[0], v1[1]};
      if (odd) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = only_finite<T>(v[e]);
      }
      acc[d] = M::mfma16(__builtin_bit_cast(vec, v), pf, acc[d]);
    }
    if (odd) {
      // A product of zero and an infinity would be a NaN, also for the rows that do not see the key: these values were left
      // out of the matrix product and go to the rows that see them one by one.
      for (int u = 0; u < kBlock; ++u) {
        if (!(odd >> (u + (u & 16)) & 1)) continue;
        const bool seen = (readable >> u & 1) && j0 + u >= my_first && j0 + u <= my_last;
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = (float)myv[u * PITCH + d * 16 + g * 4 + e];
            if (seen && !__builtin_isfinite(v)) {
#pragma unroll
              for (int dd = 0; dd < DT; ++dd)
                if (dd == d) acc[dd][e] += v;
            }
          }
      }
    }
  }
  l = sum_quarters(l);

  // The waves' results, on the scale of the largest maximum.
  if (g == 0) {
    sm[wave][col] = m;
    sl[wave][col] = l;
  }
  __syncthreads();
  float mt = kNegInf;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) mt = fmaxf(mt, sm[w][col]);
  const float own = m == kNegInf ? 0.f : pow2((m - mt) * c);
  float* const part = reinterpret_cast<float*>(vs[wave]);
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<floatx4*>(part + col * DP + d * 16 + g * 4) = m == kNegInf ? (floatx4){0, 0, 0, 0} : acc[d] * own;
  __syncthreads();
  const bool shared_out = active > 1;
  const int tile_no = (b * a.kv_heads + hk) * pl.row_tiles + tile;
  float* const ws = shared_out ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + kCounterBytes) + (size_t)tile_no * pl.chunks * part_floats<DP>() : nullptr;
  float* const mine = shared_out ? ws + (size_t)chunk_no * part_floats<DP>() : nullptr;
  const int live = min(kRows, rows - r0);

  // one float4 of the output; row `cc` of the tile
  auto put = [&](int cc, int d, floatx4 o, float lt) {
    const int rr = r0 + cc, ii = (int)fast_div((unsigned)rr, a.fd_group);
    const int tk = s.start + ii;
    if ((unsigned)tk >= (unsigned)a.tokens) return;
    const bool none = s.last(a, ii) < s.first(a, ii);
    const float inv = 1.f / lt;
    uintx2 w = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
    if (none) w = (uintx2){0, 0};
    *reinterpret_cast<uintx2*>(static_cast<T*>(a.out) + (long)tk * a.out_token + (long)(hk * a.group + rr - ii * a.group) * D + d) = w;
  };
  for (int it = tid; it < live * (DP / 4); it += kWaves * 64) {
    const int cc = it / (DP / 4), d = it % (DP / 4) * 4;
    if (d >= D) continue;
    floatx4 o = {0, 0, 0, 0};
    float mm = kNegInf, lt = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      o += *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(vs[w]) + cc * DP + d);
      mm = fmaxf(mm, sm[w][cc]);
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) lt += sm[w][cc] == kNegInf ? sl[w][cc] : sl[w][cc] * pow2((sm[w][cc] - mm) * c);
    if (!shared_out) {
      put(cc, d, o, lt);
      continue;
    }
    *reinterpret_cast<floatx4*>(mine + cc * DP + d) = o;
    if (d == 0) {
      mine[kRows * DP + cc] = mm;
      mine[kRows * DP + kRows + cc] = lt;
    }
  }
  if (!shared_out) return;

  // The workgroup that counts itself last joins the chunks.  The XCDs' L2s are not coherent with each other: the partial results are
  // released to device scope before the count and acquired after it, by one wave for the workgroup.
  __syncthreads();
  if (tid == 0) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    unsigned* cnt = static_cast<unsigned*>(a.workspace) + tile_no * 16;
    const unsigned old = atomicAdd(cnt, 1u);
    s_last = old == (unsigned)(active - 1);
    if (s_last) {
      atomicExch(cnt, 0u);
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
  }
  __syncthreads();
  if (!s_last) return;
  for (int it = tid; it < live * (DP / 4); it += kWaves * 64) {
    const int cc = it / (DP / 4), d = it % (DP / 4) * 4;
    if (d >= D) continue;
    float mm = kNegInf;
    for (int u = 0; u < active; ++u) mm = fmaxf(mm, ws[(size_t)u * part_floats<DP>() + kRows * DP + cc]);
    floatx4 o = {0, 0, 0, 0};
    float lt = 0.f;
    for (int u = 0; u < active; ++u) {
      const float* p = ws + (size_t)u * part_floats<DP>();
      const float mu = p[kRows * DP + cc], w = mu == kNegInf ? 0.f : pow2((mu - mm) * c);
      o += *reinterpret_cast<const floatx4*>(p + cc * DP + d) * w;
      lt += mu == kNegInf ? p[kRows * DP + kRows + cc] : p[kRows * DP + kRows + cc] * w;
    }
    put(cc, d, o, lt);
  }
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }

// How many workgroups the chip is given before a sequence's keys stay with one: four to a CU.
constexpr long kFill = 1024;

RowsPlan rows_plan(const AttnArgs& a, bool share) {
  RowsPlan p;
  p.row_tiles = (int)(((long)a.max_q_len * a.group + kRows - 1) / kRows);
  const long tiles = (long)a.batch * a.kv_heads * p.row_tiles;
  const int round = kWaves * kBlock;
  // the most keys between the first and the last that a tile's rows see
  const int keys = a.window > 0 && a.causal ? (int)min((long)a.max_kv_len, (long)a.window + kRows) : a.max_kv_len;
  long want = share && tiles <= kCounters ? (kFill + tiles - 1) / tiles : 1;
  const long most = max(1, (keys + round - 1) / round);
  want = min(want, most);
  const long rounds = (most + want - 1) / want;
  p.chunk = want > 1 ? (int)(rounds * round) : a.max_kv_len;
  p.chunks = want > 1 ? (int)((keys + p.chunk - 1) / p.chunk) : 1;
  return p;
}

template <typename T>
hipError_t launch_rows(const AttnArgs& a, hipStream_t st) {
  const RowsPlan p = rows_plan(a, a.workspace != nullptr);
  const dim3 grid((unsigned)(p.row_tiles * p.chunks), (unsigned)a.kv_heads, (unsigned)a.batch), block(kWaves * 64);
  switch (padded_dim(a.head_dim)) {
    case 64: hipLaunchKernelGGL((attn_rows_kernel<T, 64>), grid, block, 0, st, a, p); break;
    case 96: hipLaunchKernelGGL((attn_rows_kernel<T, 96>), grid, block, 0, st, a, p); break;
    case 128: hipLaunchKernelGGL((attn_rows_kernel<T, 128>), grid, block, 0, st, a, p); break;
    default: hipLaunchKernelGGL((attn_rows_kernel<T, 256>), grid, block, 0, st, a, p);
  }
  return hipGetLastError();
}

}  // namespace

size_t attn_workspace_bytes(const AttnArgs& a) {
  if (a.max_q_len == 0) return 0;
  const RowsPlan p = rows_plan(a, true);
  if (p.chunks <= 1) return 0;
  const size_t part = (size_t)(kRows * padded_dim(a.head_dim) + 2 * kRows) * 4;
  return kCounterBytes + (size_t)a.batch * a.kv_heads * p.row_tiles * p.chunks * part;
}

bool attn_fits(const AttnArgs& a) {
  return a.kv_heads < 65536 && a.batch < 65536 && a.max_kv_len <= 1 << 30 && (double)a.max_q_len * a.group < 2147483000.0;
}

hipError_t launch_attention(const AttnArgs& a, int dtype, hipStream_t st) {
  return dtype == T_F16 ? launch_rows<_Float16>(a, st) : launch_rows<__bf16>(a, st);
}

}  // namespace relay
