// The next token of a row:  w_i = exp((l_i - max) / T), tokens in descending order, cut off by top-k, top-p and min-p, and the one at which the
// running sum of w passes u times the sum over the kept.
//
// What is asked of the order is always a place in it: the k-th token, the one that reaches a mass.  So nothing is sorted but the few tokens
// around such a place.  Tokens are told apart by bins of equal width of their distance from the maximum, counted or added up in LDS; the bin of a place is found by
// a scan, and its tokens are gathered and sorted.  Masses are integers, multiples of 2^-S of the largest weight: sums of them have no order, and the borders between tokens are where 64 bits put them.
// A row is read three times at most in what settings commonly leave (maximum; counts or masses; gathering), from the caches after the first.
#include <float.h>

#include "decoder_ops.hpp"

namespace relay {
namespace {

constexpr int NT = 1024, WAVES = NT / 64, BINS = 2 * NT, CAP = 2048;   // threads to a row; bins of a histogram; tokens that a list holds
typedef unsigned long long u64;

template <typename T> struct Piece { typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };

// ascending with the value; +0 and -0 are one
__device__ __forceinline__ unsigned key_of(float l) {
  const int b = __builtin_bit_cast(int, l + 0.f);
  return (unsigned)b ^ ((unsigned)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) {
  return __builtin_bit_cast(float, key ^ ((unsigned)((int)~key >> 31) | 0x80000000u));
}

struct Lds {
  u64 mass[BINS];      // of a bin, then of all bins up to it
  unsigned count[BINS];
  union {
    struct {
      u64 list[CAP];   // (descending value, ascending number) as one ascending number
      u64 run[CAP];    // masses of the list up to a place
    };
    struct {
      u64 mass2[BINS];   // as above, of the digits of a crowded bin's keys (while there is no list)
      unsigned count2[BINS];
    };
  };
  double exp2s[256];   // 2^(i / 256)
  u64 wave64[WAVES];
  unsigned wave32[WAVES];
  float wavef[2][WAVES];
  int found;
  unsigned listed;
};

// Sums up to and with this thread's over the block's threads; the total.  (Two barriers: the cells are free again behind them.)
template <typename V>
__device__ __forceinline__ V block_scan(V v, V* cells, V* total) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const V o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) cells[wave] = v;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int u = 0; u < WAVES; ++u) {
    const V c = cells[u];
    if (u < wave) before += c;
    all += c;
  }
  __syncthreads();
  *total = all;
  return v + before;
}

// floor(f x) and ceil(f x), 0 <= f < 1 (of f below 2^-40 the bits past the 64th are dropped)
__device__ __forceinline__ u64 part_of(float f, u64 x) { return __umul64hi(x, (u64)((double)f * 18446744073709551616.0)); }
__device__ __forceinline__ u64 part_up(float f, u64 x) {
  const u64 m = (u64)((double)f * 18446744073709551616.0);
  return __umul64hi(x, m) + (x * m != 0);
}

template <typename T>
struct Row {
  Lds& s;
  const T* logits;
  int n, scale_bits;   // tokens; S
  float top;           // the maximum
  double per_unit;     // log2(e) / T
  float half_top, half_range, to_bin;   // distances are halved, so that none overflows
  int tid;

  // a logit as it counts: NaN as -infinity, +infinity as the largest number
  static __device__ __forceinline__ float clean(T v) { return fminf(fmaxf((float)v, -__builtin_inff()), FLT_MAX); }

  // f(logit, number) of every token; tokens of a thread in ascending order
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    constexpr int V = 16 / sizeof(T), U = 2;
    typedef typename Piece<T>::vec vec;
    const int pieces = n / V;
    for (int p0 = tid; p0 < pieces; p0 += U * NT) {
      vec v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p0 + u * NT < pieces) v[u] = *reinterpret_cast<const vec*>(logits + (size_t)(p0 + u * NT) * V);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p0 + u * NT < pieces)
#pragma unroll
          for (int e = 0; e < V; ++e) f(clean(v[u][e]), (p0 + u * NT) * V + e);
    }
    const int rest = pieces * V + tid;
    if (rest < n) f(clean(logits[rest]), rest);
  }

  __device__ __forceinline__ float distance(float l) const { return fmaf(-0.5f, l, half_top); }
  __device__ __forceinline__ bool counts(float d) const { return d <= half_range; }   // (beyond: a weight of zero)
  __device__ __forceinline__ int bin(float d) const { return min((int)(d * to_bin), BINS - 1); }
  __device__ __forceinline__ double exponent(float l) const { return ((double)l - (double)top) * per_unit; }
  // 2^z: z = i / 256 + r, a table and the series of 2^r to the fourth power (|r| <= 2^-9: off by 2^-54)
  __device__ __forceinline__ double pow2(double z) const {
    const double magic = 6755399441055744.0;   // 1.5 2^52: what is added to it is rounded to a whole number
    const double t = fma(z, 256.0, magic);
    const int i = (int)(unsigned)__builtin_bit_cast(u64, t);
    const double r = fma(t - magic, -1.0 / 256, z);
    const double p = fma(fma(fma(fma(9.6181291076284771619791e-3, r, 5.5504108664821579953143e-2), r, 0.24022650695910071233355), r, 0.69314718055994530941723), r, 1.0);
    return ldexp(p * s.exp2s[i & 255], i >> 8);
  }
  // as a multiple of 2^-S, rounded
  __device__ __forceinline__ u64 weight(float l) const {
    const double w = ldexp(pow2(exponent(l)), scale_bits) + 4503599627370496.0;   // (at most 2^51; 2^52 + w has w as its lowest bits)
    return __builtin_bit_cast(u64, w) & 0x000fffffffffffffull;
  }

  // Bins' counts into s.count and, if asked for, masses into s.mass, each then with those of all bins ahead of it; the totals.
  __device__ __forceinline__ void histogram(bool masses, unsigned* total_count, u64* total_mass) {
    for (int i = tid; i < BINS; i += NT) s.count[i] = 0, s.mass[i] = 0;
    __syncthreads();
    each([&](float l, int) {
      const float d = distance(l);
      if (counts(d)) {
        const int b = bin(d);
        atomicAdd(&s.count[b], 1u);
        if (masses) atomicAdd(&s.mass[b], weight(l));
      }
    });
    __syncthreads();
    scan_bins(s.count, s.mass, total_count, total_mass);
  }
  __device__ __forceinline__ void scan_bins(unsigned* count, u64* mass, unsigned* total_count, u64* total_mass) {
    const unsigned a = count[2 * tid], b = count[2 * tid + 1], end = block_scan<unsigned>(a + b, s.wave32, total_count);
    count[2 * tid] = end - b;
    count[2 * tid + 1] = end;
    const u64 c = mass[2 * tid], d = mass[2 * tid + 1], mass_end = block_scan<u64>(c + d, s.wave64, total_mass);
    mass[2 * tid] = mass_end - d;
    mass[2 * tid + 1] = mass_end;
    __syncthreads();
  }
  // the first of `size` running sums that reaches (OVER: passes) a goal; it must be there
  template <bool OVER, typename V>
  __device__ __forceinline__ int first_of(const V* sums, int size, V goal) {
    for (int i = tid; i < size; i += NT) {
      const V at = sums[i], before = i ? sums[i - 1] : 0;
      if (OVER ? at > goal && before <= goal : at >= goal && (i == 0 || before < goal)) s.found = i;
    }
    __syncthreads();
    const int r = s.found;
    __syncthreads();
    return r;
  }

  // The tokens that `wanted` names, sorted, with their running masses; how many, or more than CAP if they do not fit.
  template <typename F>
  __device__ __forceinline__ int gather(F wanted) {
    if (tid == 0) s.listed = 0;
    __syncthreads();
    each([&](float l, int i) {
      if (wanted(l)) {
        const unsigned at = atomicAdd(&s.listed, 1u);
        if (at < CAP) s.run[at] = (u64)~key_of(l) << 32 | (unsigned)i;
      }
    });
    __syncthreads();
    const int m = (int)min(s.listed, (unsigned)CAP + 1);
    if (m > CAP) {
      __syncthreads();
      return m;
    }
    // up to 512: each token counts those ahead of it, several threads to a token; more: by exchanges
    if (m <= 512) {
      int per = 1;   // threads to a token
      while (2 * per * m <= NT && per < 64) per *= 2;
      const int t = tid / per, sub = tid & (per - 1);
      int ahead = 0;
      const u64 mine = t < m ? s.run[t] : 0;
      if (t < m)
        for (int j = sub; j < m; j += per) ahead += s.run[j] < mine;
      for (int d = 1; d < per; d <<= 1) ahead += __shfl_xor(ahead, d);
      if (t < m && sub == 0) s.list[ahead] = mine;
    } else {
      for (int i = tid; i < CAP; i += NT) s.list[i] = i < m ? s.run[i] : ~0ull;
      int size = 1024;
      if (m > 1024) size = 2048;
      for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
          __syncthreads();
          for (int h = tid; h < size / 2; h += NT) {
            const int a = 2 * h - (h & (j - 1)), b = a + j;   // (a: h with a zero put in at bit j)
            const u64 x = s.list[a], y = s.list[b];
            if ((x > y) == ((a & k) == 0)) {
              s.list[a] = y;
              s.list[b] = x;
            }
          }
        }
    }
    __syncthreads();
    // two neighbours to a thread
    u64 total;
    const u64 a = 2 * tid < m ? weight(listed(2 * tid)) : 0, b = 2 * tid + 1 < m ? weight(listed(2 * tid + 1)) : 0;
    const u64 end = block_scan<u64>(a + b, s.wave64, &total);
    s.run[2 * tid] = end - b;
    s.run[2 * tid + 1] = end;
    __syncthreads();
    return m;
  }
  __device__ __forceinline__ float listed(int i) const { return value_of(~(unsigned)(s.list[i] >> 32)); }
  __device__ __forceinline__ int number(int i) const { return (int)(unsigned)s.list[i]; }

  enum Goal { RANK, REACH, PASS };
  struct Place { u64 mass; int number; float logit; };   // of the tokens up to the place, with its own; the token there (PASS)

  // A place within bin b: its goal-th token (RANK), or the first at which the bin's masses reach or pass `goal`.
  __device__ __forceinline__ Place within(int b, Goal kind, u64 goal) {
    unsigned prefix = 0;
    int shift = 32;
    u64 base = 0;
    for (;;) {
      const int m = gather([&](float l) {
        const float d = distance(l);
        return counts(d) && bin(d) == b && (shift == 32 || key_of(l) >> shift == prefix);
      });
      if (m <= CAP) {
        const int i = kind == RANK ? (int)goal - 1 : kind == REACH ? first_of<false>(s.run, m, goal) : first_of<true>(s.run, m, goal);
        return {base + s.run[i], number(i), listed(i)};
      }
      if (shift == 0) break;
      // too many: told apart by the next digit of their keys
      const int digits = shift == 10 ? 10 : 11, next = shift - digits, mask = (1 << digits) - 1;
      for (int i = tid; i < BINS; i += NT) s.count2[i] = 0, s.mass2[i] = 0;
      __syncthreads();
      each([&](float l, int) {
        const float d = distance(l);
        const unsigned key = key_of(l);
        if (counts(d) && bin(d) == b && (shift == 32 || key >> shift == prefix)) {
          const int digit = mask - (int)(key >> next & (unsigned)mask);   // (descending)
          atomicAdd(&s.count2[digit], 1u);
          atomicAdd(&s.mass2[digit], weight(l));
        }
      });
      __syncthreads();
      unsigned tc;
      u64 tm;
      scan_bins(s.count2, s.mass2, &tc, &tm);
      const int at = kind == RANK ? first_of<false>(s.count2, BINS, (unsigned)goal)
                                  : kind == REACH ? first_of<false>(s.mass2, BINS, goal) : first_of<true>(s.mass2, BINS, goal);
      const u64 ahead = at ? s.mass2[at - 1] : 0;
      goal -= kind == RANK ? (u64)(at ? s.count2[at - 1] : 0) : ahead;
      base += ahead;
      prefix = (shift == 32 ? 0 : prefix << digits) | (unsigned)(mask - at);
      shift = next;
      __syncthreads();
    }
    // more tokens of one value than a list holds
    const float l = value_of(prefix);
    const u64 w = weight(l);
    const u64 which = kind == RANK ? goal : kind == REACH ? (goal + w - 1) / w : goal / w + 1;
    int num = 0;
    if (kind == PASS) {   // each thread counts a run of its own
      const int run = (n + NT - 1) / NT, lo = min(tid * run, n), hi = min(lo + run, n);
      unsigned mine = 0, total;
      for (int i = lo; i < hi; ++i) mine += key_of(clean(logits[i])) == prefix;
      const unsigned end = block_scan<unsigned>(mine, s.wave32, &total);
      if (end >= which && end - mine < which) {
        unsigned at = end - mine;
        for (int i = lo; i < hi; ++i)
          if (key_of(clean(logits[i])) == prefix && ++at == which) s.found = i;
      }
      __syncthreads();
      num = s.found;
      __syncthreads();
    }
    return {base + which * w, num, l};
  }
  // a place among all tokens, from the bins' running sums
  __device__ __forceinline__ Place among(Goal kind, u64 goal) {
    const int b = kind == RANK ? first_of<false>(s.count, BINS, (unsigned)goal)
                               : kind == REACH ? first_of<false>(s.mass, BINS, goal) : first_of<true>(s.mass, BINS, goal);
    const u64 ahead = b ? s.mass[b - 1] : 0;
    Place p = within(b, kind, goal - (kind == RANK ? (u64)(b ? s.count[b - 1] : 0) : ahead));
    p.mass += ahead;
    return p;
  }
};

template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(const SampleArgs a) {
  __shared__ Lds s;
  const int r = (int)blockIdx.x, tid = (int)threadIdx.x, wave = tid >> 6;
  Row<T> row{s, static_cast<const T*>(a.logits) + (size_t)r * a.logits_stride, a.vocab, a.scale_bits};
  row.tid = tid;
  // settings, those that are off as such
  float temperature = a.temperature ? a.temperature[r] : 1.f, top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
  float u = a.uniform ? a.uniform[r] : 0.f;
  int top_k = a.top_k ? a.top_k[r] : 0;
  if (!(temperature == temperature)) temperature = 1.f;
  if (top_k <= 0 || top_k >= a.vocab) top_k = 0;
  const bool cut_p = top_p < 1.f, cut_min = min_p > 0.f;
  min_p = fminf(min_p, 1.f);
  u = fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);   // (a NaN: 0)
  const bool greedy = !a.uniform || temperature <= 0.f || top_k == 1 || top_p <= 0.f;

  // the maximum, the first token that has it, the lowest logit
  float best = -__builtin_inff(), low = __builtin_inff();
  int at = a.vocab;
  row.each([&](float l, int i) {
    if (l > best) best = l, at = i;
    if (l >= -FLT_MAX) low = fminf(low, l);
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float o = __shfl_xor(best, d);
    const int oi = __shfl_xor(at, d);
    if (o > best || (o == best && oi < at)) best = o, at = oi;
    low = fminf(low, __shfl_xor(low, d));
  }
  if ((tid & 63) == 0) s.wavef[0][wave] = best, s.wavef[1][wave] = low, s.wave32[wave] = (unsigned)at;
  if (tid < 256) s.exp2s[tid] = exp2(tid / 256.0);
  __syncthreads();
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const float o = s.wavef[0][v];
    const int oi = (int)s.wave32[v];
    if (o > best || (o == best && oi < at)) best = o, at = oi;
    low = fminf(low, s.wavef[1][v]);
  }
  __syncthreads();
  if (best == -__builtin_inff() || greedy) {
    if (tid == 0) {
      const bool any = best > -__builtin_inff();
      a.tokens[r] = any ? at : -1;
      if (a.probs) a.probs[r] = any ? 1.f : 0.f;
    }
    return;
  }
  row.top = best;
  row.per_unit = 1.4426950408889634074 / (double)temperature;
  row.half_top = 0.5f * best;
  const double reach = 0.5 * (a.scale_bits + 1.0) / row.per_unit;   // where weights of half a unit lie
  row.half_range = (float)fmin(reach, (double)fminf(0.5f * best - 0.5f * low, FLT_MAX));
  row.to_bin = (float)BINS / row.half_range;
  if (!(row.to_bin < 1e30f)) row.to_bin = 0.f;

  const double z_min = cut_min ? log2((double)min_p) : 0.0;
  auto likely = [&](float l) { return row.exponent(l) >= z_min; };
  unsigned tokens = 0;
  u64 total = 0, goal_p = 0;
  int listed = CAP + 1;                            // tokens in the list, if it holds all that can be kept
  bool by_value = !top_k && !cut_p && cut_min;     // ... which then are those that min-p leaves
  for (bool masses = !top_k;;) {
    int last_bin = -1;                             // ... or those of the bins up to this
    if (!by_value) {
      row.histogram(masses, &tokens, &total);
      if (top_k && (unsigned)top_k >= tokens) {    // (the rest have no weight)
        top_k = 0;
        by_value = !cut_p && cut_min;
        if (!masses) {
          masses = true;
          continue;
        }
      }
      if (top_k || cut_p) {
        int b;
        if (top_k) {
          b = row.template first_of<false>(s.count, BINS, (unsigned)top_k);
        } else {
          goal_p = part_up(top_p, total);
          goal_p = goal_p ? goal_p : 1;
          b = row.template first_of<false>(s.mass, BINS, goal_p);
        }
        if (s.count[b] <= CAP) last_bin = b;
      }
    }
    if (by_value || last_bin >= 0)
      listed = row.gather([&](float l) {
        const float d = row.distance(l);
        return row.counts(d) && (by_value ? likely(l) : row.bin(d) <= last_bin);
      });
    if (listed <= CAP || (masses && !by_value)) break;
    by_value = false;
    masses = true;
  }
  if (top_k && listed <= CAP) listed = min(listed, top_k);
  u64 kept = total;
  int token = 0;
  float logit = best;
  if (listed <= CAP) {
    // all that can be kept stands in the list, in order
    if (cut_p) {
      if (!goal_p) goal_p = part_up(top_p, s.run[listed - 1]);
      goal_p = goal_p ? goal_p : 1;
      listed = min(listed, row.template first_of<false>(s.run, listed, goal_p) + 1);
    }
    if (cut_min) {   // (the first of the list always stays)
      for (int i = tid; i < listed; i += NT)
        if (likely(row.listed(i)) && (i + 1 == listed || !likely(row.listed(i + 1)))) s.found = i;
      __syncthreads();
      listed = s.found + 1;
      __syncthreads();
    }
    kept = s.run[listed - 1];
    const int i = row.template first_of<true>(s.run, listed, part_of(u, kept));
    token = row.number(i);
    logit = row.listed(i);
  } else {
    for (int step = 0; step < 4; ++step) {
      if ((step == 0 && !top_k) || (step == 1 && !cut_p) || (step == 2 && !cut_min)) continue;
      if (step == 2) {
        u64 mine = 0, sum;
        row.each([&](float l, int) { if (row.counts(row.distance(l)) && likely(l)) mine += row.weight(l); });
        block_scan<u64>(mine, s.wave64, &sum);
        kept = sum < kept ? sum : kept;
        continue;
      }
      const u64 up = part_up(top_p, kept);
      const auto place = row.among(step == 0 ? Row<T>::RANK : step == 1 ? Row<T>::REACH : Row<T>::PASS,
                                   step == 0 ? (u64)top_k : step == 1 ? (up ? up : 1) : part_of(u, kept));
      if (step < 3) {
        kept = place.mass;
      } else {
        token = place.number;
        logit = place.logit;
      }
    }
  }
  if (tid == 0) {
    a.tokens[r] = token;
    if (a.probs) a.probs[r] = (float)(row.pow2(row.exponent(logit)) / ldexp((double)kept, -a.scale_bits));
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& args, int dtype, hipStream_t st) {
  SampleArgs a = args;
  int bits = 0;   // vocab <= 2^bits
  while ((1 << bits) < a.vocab) ++bits;
  a.scale_bits = 62 - bits < 51 ? 62 - bits : 51;
  const dim3 grid((unsigned)a.rows), block(NT);
  if (dtype == T_F16) hipLaunchKernelGGL((sample_kernel<_Float16>), grid, block, 0, st, a);
  else if (dtype == T_BF16) hipLaunchKernelGGL((sample_kernel<__bf16>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((sample_kernel<float>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace relay
