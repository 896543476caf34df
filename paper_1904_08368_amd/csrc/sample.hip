// The next token of a row:  w_i = exp((l_i - max) / T), tokens in descending order, cut off by top-k, top-p and min-p, and the one at which the
// running sum of w passes u times the sum over the kept.
//
// What is asked of the order is always a place in it: the k-th token, the one that reaches a mass.  So nothing is sorted but the few tokens
// around such places.  Tokens are told apart by bins of equal width of their distance from the maximum, counted or added up in LDS.  A place lies in one bin; the mass that the places behind
// it start from is known up to that bin's, which leaves them few bins.  All these bins' tokens are gathered and sorted, and give the places exactly.
// Masses are integers, multiples of 2^-S of the largest weight: sums of them have no order, and the borders between tokens are where 64 bits put them.
// So a row is read three times: maximum; counts or masses; gathering.  One workgroup reads it where there are many rows, from the caches after the first time.  Of few rows each is shared out over
// workgroups, a launch to each reading.
// One row of 128000 fp16, top-k 50 and top-p: 16.5 us, launches of 4, 2.5 and 11 that wait for memory and for each other.  48 rows of 151643 bf16, top-p: 49 us, of 7, 14 and 29: weights in 64 bits and
// additions to LDS in the second (50 % and 28 % of the clocks), in the third a last workgroup that sorts some 300 tokens of one value.  256 rows of 50257 fp32, each with its own settings: 48 us,
// additions to LDS (some 30 clocks for a wave's, whose lanes meet on banks) and weights by eight waves a CU.
#include <float.h>

#include "decoder_ops.hpp"
#include "wave_ops.hpp"

namespace relay {
namespace {

constexpr int BINS = 2048, CAP = 2048;   // of a histogram; tokens that a list holds
constexpr int NT = 512, WAVES = NT / 64; // threads of a workgroup (of 1024 each would have too few registers)
constexpr int PARTS = 32;                // workgroups that share a row at most
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
  u64 mass[BINS];        // of a bin, then of all bins up to it
  unsigned count[BINS];
  unsigned place[BINS];  // of a bin's tokens in the list
  unsigned char gathered[BINS];
  union {
    struct {
      alignas(16) u64 list[CAP];   // (descending value, ascending number) as one ascending number
      alignas(16) u64 run[CAP];    // masses of all tokens up to a place of the list
    };
    struct {
      u64 mass2[BINS];   // as above, of the digits of a crowded bin's keys (while there is no list)
      unsigned count2[BINS];
    };
  };
  double exp2s[256];     // 2^(i / 256)
  u64 wave64[WAVES];
  unsigned wave32[WAVES];
  float wavef[2][WAVES];
  int found;
  unsigned listed;
};

// floor(f x) and ceil(f x), 0 <= f < 1 (of f below 2^-40 the bits past the 64th are dropped)
__device__ __forceinline__ u64 part_of(float f, u64 x) { return __umul64hi(x, (u64)((double)f * 18446744073709551616.0)); }
__device__ __forceinline__ u64 part_up(float f, u64 x) {
  const u64 m = (u64)((double)f * 18446744073709551616.0);
  return __umul64hi(x, m) + (x * m != 0);
}

__device__ const float kNothing = 0.f;
// A row's settings; those that are off as such.
struct Settings {
  float temperature, top_p, min_p, u;
  int top_k;
  bool cut_p, cut_min, greedy;
  double z_min;
  __device__ Settings(const SampleArgs& a, int r) {
    // (all asked for at once; what is not there is read from the uniform numbers, and not used.  Without these the first is what is asked for, whatever the rest.)
    const float* const some = a.uniform ? a.uniform : &kNothing;
    const int at = a.uniform ? r : 0;
    const float t = (a.temperature ? a.temperature : some)[at], p = (a.top_p ? a.top_p : some)[at], m = (a.min_p ? a.min_p : some)[at], v = some[at];
    const int k = (a.top_k ? a.top_k : reinterpret_cast<const int32_t*>(some))[at];
    temperature = a.temperature ? t : 1.f;
    top_p = a.top_p ? p : 1.f;
    min_p = a.min_p ? m : 0.f;
    u = v;
    top_k = a.top_k ? k : 0;
    if (!(temperature == temperature)) temperature = 1.f;
    if (top_k <= 0 || top_k >= a.vocab) top_k = 0;
    cut_p = top_p < 1.f;
    cut_min = min_p > 0.f;
    u = fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);   // (a NaN: 0)
    greedy = !a.uniform || temperature <= 0.f || top_k == 1 || top_p <= 0.f || min_p > 1.f;   // (no w is above 1)
    z_min = cut_min ? log2((double)min_p) : 0.0;
  }
  // What the second reading adds up: nothing, where the third finds all that min-p keeps by itself, or all that top-k keeps from some `maxima` of parts of the row: as many of them as top-k asks for
  // bound its tokens from below.  Otherwise bins' tokens, for top-k, and their masses.
  __device__ bool by_value() const { return !top_k && !cut_p && cut_min; }
  __device__ bool by_maxima(int maxima) const { return top_k && 2 * top_k <= maxima; }   // (more of them and the bound lies low)
  __device__ bool masses() const { return !top_k || top_k > CAP / 2; }   // (of a few tokens the list tells)
};

// the same in all lanes: kept once
__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }

__device__ __forceinline__ double uniform(double v) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(double, (u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)b));
}

struct Top { float best, low; int at; };   // the maximum, the lowest number, the first token that has the maximum
__device__ __forceinline__ void merge(Top& t, float best, float low, int at) {
  if (best > t.best || (best == t.best && at < t.at)) t.best = best, t.at = at;
  t.low = fminf(t.low, low);
}
__device__ __forceinline__ Top of_wave(const Top& t) {   // all lanes'
  const float best = wave_fold32(t.best, [](float x, float y) { return fmaxf(x, y); });
  return {best, wave_fold32(t.low, [](float x, float y) { return fminf(x, y); }), wave_fold32(t.best == best ? t.at : 0x7fffffff, [](int x, int y) { return min(x, y); })};
}

template <typename T>
struct Row {
  Lds& s;
  const T* logits;
  int n, scale_bits;   // tokens; S
  int piece0, piece1;  // the 16-byte pieces that this workgroup reads,
  bool tail;           // ... and whether what is left behind the last whole one
  int tid;
  float top;           // the maximum
  double per_unit;     // log2(e) / T
  float half_top, half_range, to_bin;   // distances are halved, so that none overflows
  float own;           // the maximum of what this thread has read
  struct Bins { int first, last; };
  Bins of_k, of_p, of_min, of_u;        // what is gathered: the bins where top-k, top-p and min-p cut, and where the token is

  __device__ Row(Lds& lds, const SampleArgs& a, int r) : s(lds), logits(static_cast<const T*>(a.logits) + (size_t)r * a.logits_stride), n(a.vocab), scale_bits(a.scale_bits),
      piece0(0), piece1(a.vocab / V), tail(true), tid((int)threadIdx.x), of_k{BINS, BINS}, of_p{BINS, BINS}, of_min{BINS, BINS}, of_u{BINS, BINS} {}
  __device__ void share(int g, int parts) {
    const int pieces = n / V;
    piece0 = (int)((long)pieces * g / parts);
    piece1 = (int)((long)pieces * (g + 1) / parts);
    tail = g == parts - 1;
  }

  static constexpr int V = 16 / sizeof(T);
  typedef typename Piece<T>::vec vec;

  // f(logit, number) of every token, those of a thread in ascending order; 2 U pieces on their way.  (A NaN is as far from the maximum as nothing else, and has no weight;
  // +infinity counts as the largest number.)
  template <int U>
  __device__ __forceinline__ void load(vec (&v)[U], int p) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p + u * NT < piece1) v[u] = *reinterpret_cast<const vec*>(logits + (size_t)(p + u * NT) * V);
  }
  template <int U, typename F>
  __device__ __forceinline__ void each(F f) const {
    vec now[U];
    load(now, piece0 + tid);
    each(f, now);
  }
  // ... the first U of this thread being there
  template <int U, typename F>
  __device__ __forceinline__ void each(F f, vec (&now)[U]) const {
    pieces([&](const vec& v, int i) {
#pragma unroll
      for (int e = 0; e < V; ++e) f((float)v[e], i + e);
    }, [&](float l, int i) { f(l, i); }, now);
  }
  // f(piece, number of its first token) of every piece, one(logit, number) of what is left behind the last whole one
  template <int U, typename F, typename G>
  __device__ __forceinline__ void pieces(F f, G one, vec (&now)[U]) const {
    vec next[U];
    for (int p = piece0 + tid; p < piece1; p += U * NT) {
      load(next, p + U * NT);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u * NT < piece1) f(now[u], (p + u * NT) * V);
        now[u] = next[u];
      }
    }
    const int rest = n / V * V + tid;
    if (tail && rest < n) one((float)logits[rest], rest);
  }

  // Sums up to and with this lane's over the wave: within rows of 16 lanes, then the rows' last lanes to the rows behind.
  template <int CTRL, int ROWS>
  static __device__ __forceinline__ unsigned moved(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
  template <int CTRL, int ROWS>
  static __device__ __forceinline__ u64 moved(u64 v) { return (u64)moved<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | moved<CTRL, ROWS>((unsigned)v); }
  template <typename N>
  static __device__ __forceinline__ N wave_scan(N v) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
  }
  // The same over the block's threads; the total.  (Two barriers: the cells are free again behind them.)
  template <typename N>
  __device__ __forceinline__ N scan(N v, N* cells, N* total) const {
    const int lane = tid & 63, wave = tid >> 6;
    v = wave_scan(v);
    if (lane == 63) cells[wave] = v;
    __syncthreads();
    N before = 0, all = 0;
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      const N c = cells[u];
      if (u < wave) before += c;
      all += c;
    }
    __syncthreads();
    *total = all;
    return v + before;
  }
  // `size` numbers become their running sums, SIZE / NT neighbours to a thread
  template <int SIZE, typename N>
  __device__ __forceinline__ void running(N* v, N* cells, N* total) const {
    constexpr int PER = SIZE / NT;
    N mine[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      mine[i] = v[tid * PER + i];
      sum += mine[i];
    }
    N at = scan<N>(sum, cells, total) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      at += mine[i];
      v[tid * PER + i] = at;
    }
    __syncthreads();
  }
  // the first of `size` running sums that reaches (OVER: passes) a goal, or the last; each wave looks for itself, a range of 64th parts at a time
  template <bool OVER, typename N>
  __device__ __forceinline__ int first_of(const N* sums, int size, N goal) const {
    int lo = 0;   // all ahead of this lie below the goal
    for (int step = size; step > 1;) {
      const int len = min(step, size - lo);
      step = (len + 63) / 64;
      const int at = min(lo + ((tid & 63) + 1) * step, size) - 1;
      const unsigned long long there = __ballot(OVER ? sums[at] > goal : sums[at] >= goal);
      lo = min(lo + (there ? __builtin_ctzll(there) : 63) * step, size - 1);
    }
    return lo;
  }

  // ---- the maximum
  // The first token that has it where that is what is asked for; else the lowest number, which keeps the bins narrow.  -infinity among the logits hides it, unless the temperature is high and the bins
  // were wide without it.
  __device__ __forceinline__ Top extremes(const Settings& s0) {
    Top t{-__builtin_inff(), __builtin_inff(), n};
    if (s0.greedy) {
      each<2>([&](float l, int i) { if (l > t.best) t.best = l, t.at = i; });
    } else if (s0.temperature > 4.f) {
      each<2>([&](float l, int) {
        t.best = fmaxf(t.best, l);
        t.low = l >= -FLT_MAX ? fminf(t.low, l) : t.low;
      });
    } else {
      each<4>([&](float l, int) {
        t.best = fmaxf(t.best, l);
        t.low = fminf(t.low, l);
      });
    }
    own = t.best;
    t = of_wave(t);
    if ((tid & 63) == 0) s.wavef[0][tid >> 6] = t.best, s.wavef[1][tid >> 6] = t.low, s.wave32[tid >> 6] = (unsigned)t.at;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) merge(t, s.wavef[0][w], s.wavef[1][w], (int)s.wave32[w]);
    __syncthreads();
    return t;
  }
  __device__ __forceinline__ void set(const Top& t, float temperature) {
    top = fminf(t.best, FLT_MAX);
    per_unit = 1.4426950408889634074 / (double)temperature;
    half_top = 0.5f * top;
    const double reach = 0.5 * (scale_bits + 1.0) / per_unit;   // where weights of half a unit lie
    half_range = (float)fmin(reach, (double)fminf(0.5f * top - 0.5f * fmaxf(t.low, -FLT_MAX), FLT_MAX));
    to_bin = (float)BINS / half_range;
    if (!(to_bin < 1e30f)) to_bin = 0.f;
    top = uniform(top), half_top = uniform(half_top), half_range = uniform(half_range), to_bin = uniform(to_bin), per_unit = uniform(per_unit);
    for (int i = tid; i < 256; i += NT) s.exp2s[i] = exp2(i / 256.0);
    __syncthreads();
  }

  // ---- weights
  __device__ __forceinline__ float distance(float l) const { return fmaf(-0.5f, l, half_top); }
  __device__ __forceinline__ bool weighs(float d) const { return d <= half_range; }   // (beyond: a weight of zero)
  __device__ __forceinline__ int bin(float d) const { return max(min((int)(d * to_bin), BINS - 1), 0); }
  __device__ __forceinline__ double exponent(float l) const { return ((double)fminf(l, top) - (double)top) * per_unit; }
  // 2^z: z = i / 256 + r, a table and the series of 2^r to the fourth power (|r| <= 2^-9: off by 2^-54)
  __device__ __forceinline__ double pow2(double z, int up = 0) const {   // (2^(z + up))
    const double magic = 6755399441055744.0;   // 1.5 2^52: what is added to it is rounded to a whole number
    const double t = fma(z, 256.0, magic);
    const int i = (int)(unsigned)__builtin_bit_cast(u64, t);
    const double r = fma(t - magic, -1.0 / 256, z);
    const double p = fma(fma(fma(fma(9.6181291076284771619791e-3, r, 5.5504108664821579953143e-2), r, 0.24022650695910071233355), r, 0.69314718055994530941723), r, 1.0);
    return ldexp(p * s.exp2s[i & 255], (i >> 8) + up);
  }
  // as a multiple of 2^-S, rounded
  __device__ __forceinline__ u64 weight(float l) const {
    const double w = pow2(exponent(l), scale_bits) + 4503599627370496.0;   // (at most 2^51; 2^52 + w has w as its lowest bits)
    return __builtin_bit_cast(u64, w) & 0x000fffffffffffffull;
  }

  // ---- bins
  __device__ __forceinline__ void clear_bins() const {
    for (int i = tid; i < BINS; i += NT) s.count[i] = 0, s.mass[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void fill_bins(bool counts, bool masses) const {
    vec first[1];
    load(first, piece0 + tid);
    fill_bins(counts, masses, first);
  }
  // (A piece's bins and weights side by side, and only then what is added to them: one behind the other they would wait for each other's table entries.)
  __device__ __forceinline__ void fill_bins(bool counts, bool masses, vec (&first)[1]) const {
    auto add = [&](float d, int b, u64 w) {
      if (weighs(d)) {
        if (counts) atomicAdd(&s.count[b], 1u);
        if (masses) atomicAdd(&s.mass[b], w);
      }
    };
    pieces([&](const vec& v, int) {
      float d[V];
      int b[V];
      u64 w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        d[e] = distance((float)v[e]);
        b[e] = bin(d[e]);
      }
      if (masses) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          w[e] = weight((float)v[e]);
          if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (four at a time: eight take too many registers)
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) add(d[e], b[e], w[e]);
    }, [&](float l, int) { add(distance(l), bin(distance(l)), weight(l)); }, first);
    __syncthreads();
  }

  // ---- the list
  __device__ __forceinline__ bool wanted(int b) const {
    auto in = [b](const Bins& r) { return (int)((unsigned)(b - r.first) <= (unsigned)(r.last - r.first)); };
    return (in(of_k) | in(of_p) | in(of_min) | in(of_u)) != 0;
  }
  __device__ __forceinline__ float listed(int i) const { return value_of(~(unsigned)(s.list[i] >> 32)); }
  __device__ __forceinline__ int number(int i) const { return (int)(unsigned)s.list[i]; }
  static __device__ __forceinline__ u64 entry(float l, int i) { return (u64)~key_of(l) << 32 | (unsigned)i; }
  // Two ranges of logits that hold all that is gathered and little else: of few tokens more is then asked.
  struct Near {
    float at0, reach0, at1, reach1;
    __device__ __forceinline__ bool operator()(float l) const { return ((int)(fabsf(fmaf(-0.5f, l, at0)) <= reach0) | (int)(fabsf(fmaf(-0.5f, l, at1)) <= reach1)) != 0; }
  };
  // tokens at distances a .. b, which are found again with a rounding or two of their own
  __device__ __forceinline__ void around(float a, float b, float* at, float* reach) const {
    *at = half_top - 0.5f * (a + b);
    *reach = 0.5f * (b - a) + 1e-6f * (fabsf(half_top) + b);
    if (!(fabsf(*at) < FLT_MAX) || !(*reach < FLT_MAX) || top == FLT_MAX || to_bin == 0.f) *at = 0.f, *reach = __builtin_inff();   // (all of them: also where bins have no width, and the first holds all)
    *at = uniform(*at), *reach = uniform(*reach);
  }
  __device__ __forceinline__ Near near_bins() const {
    auto none = [](const Bins& r) { return r.first >= BINS; };
    int first = BINS, last = -1;
    if (!none(of_k)) first = min(first, of_k.first), last = max(last, of_k.last);
    if (!none(of_p)) first = min(first, of_p.first), last = max(last, of_p.last);
    if (!none(of_min)) first = min(first, of_min.first), last = max(last, of_min.last);
    const float width = half_range / (float)BINS;
    Near n;
    around((float)of_u.first * width, (float)(of_u.last + 1) * width, &n.at0, &n.reach0);
    n.at1 = n.at0, n.reach1 = n.reach0;
    if (last >= 0) {
      around((float)first * width, (float)(last + 1) * width, &n.at1, &n.reach1);
      if (none(of_u)) n.at0 = n.at1, n.reach0 = n.reach1;
    }
    return n;
  }
  __device__ __forceinline__ Near near_value(double z_min) const {
    Near n;
    around(0.f, (float)fmin(-0.5 * z_min / per_unit, 2.0 * (double)half_range), &n.at0, &n.reach0);
    n.at1 = n.at0, n.reach1 = n.reach0;
    return n;
  }
  __device__ __forceinline__ int gather_bins(vec (&first)[2]) const {
    return gather(near_bins(), [&](float l) { return of_bins(l); }, first);
  }
  __device__ __forceinline__ int gather_value(double z_min, vec (&first)[2]) const {
    return gather(near_value(z_min), [&](float l) { return of_value(l, z_min); }, first);
  }
  // The tokens that `is` names, of those that `near` does, into s.run, as they come; how many, or more than CAP if they do not fit.
  template <typename N, typename F>
  __device__ __forceinline__ int gather(N near, F is, vec (&first)[2]) const {
    constexpr bool NEAR = V > 4;   // (of four tokens to a piece, a wave waits more often for one that is near than it saves: without / with, 256 rows of 50257 in fp32 50 / 58 us; bf16, 64 x 128000 36 / 32)
    if (tid == 0) s.listed = 0;
    __syncthreads();
    auto take = [&](float l, int i) {
      const unsigned at = atomicAdd(&s.listed, 1u);
      if (at < CAP) s.run[at] = entry(l, i);
    };
    pieces([&](const vec& v, int i) {
      unsigned hits = 0;
#pragma unroll
      for (int e = 0; e < V; ++e) hits |= (unsigned)(NEAR ? near((float)v[e]) : is((float)v[e])) << e;
      for (; hits; hits &= hits - 1) {   // (one place of code for all of a piece's: eight took too many registers)
        const int e = __builtin_ctz(hits);
        float l = (float)v[0];
#pragma unroll
        for (int j = 1; j < V; ++j) l = e == j ? (float)v[j] : l;
        if (!NEAR || is(l)) take(l, i + e);
      }
    }, [&](float l, int i) { if (is(l)) take(l, i); }, first);
    __syncthreads();
    return (int)min(s.listed, (unsigned)CAP + 1);
  }
  // is a token one of the bins that are gathered (or, by its value, one that min-p leaves)?
  __device__ __forceinline__ bool of_bins(float l) const {
    const float d = distance(l);
    return (int)s.gathered[bin(d)] & (int)weighs(d);
  }
  __device__ __forceinline__ bool of_value(float l, double z_min) const { return (int)(exponent(l) >= z_min) & (int)weighs(distance(l)); }
  // how many of `len` numbers (a multiple of 8) from `from` on, 16-byte aligned, are less than `mine`
  static __device__ __forceinline__ int less(const u64* from, int len, u64 mine) {
    typedef u64 pair __attribute__((ext_vector_type(2)));
    int n = 0;
    for (int j = 0; j < len; j += 8) {
      pair v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const pair*>(from + j + 2 * i);
#pragma unroll
      for (int i = 0; i < 4; ++i) n += (v[i][0] < mine) + (v[i][1] < mine);
    }
    return n;
  }
  // s.run in order into s.list, then the masses of all tokens up to each.  Each token looks for its place: up to 128 among all; up to 512 among those of its bin, which are brought together
  // first.  More are sorted by exchanges.
  // masses: s.mass holds the bins' running masses, and the list may have gaps; else it begins with the first of all tokens and has none.
  __device__ __forceinline__ void sort(int m, bool masses) const {
    auto bin_of = [&](u64 v) { return bin(distance(value_of(~(unsigned)(v >> 32)))); };
    if (m <= NT) {
      const bool together = m > 128;
      u64* const from = together ? s.list : s.run;
      for (int i = tid; i < 8 * 64; i += NT) from[m + i] = ~0ull;   // (what is read behind the last, and is not less than any)
      if (together) {
        for (int b = tid; b < BINS; b += NT) s.place[b] = 0;
        __syncthreads();
        if (tid < m) atomicAdd(&s.place[bin_of(s.run[tid])], 1u);
        __syncthreads();
        unsigned all;
        running<BINS>(s.place, s.wave32, &all);
        if (tid < m) {
          const u64 v = s.run[tid];
          s.list[atomicSub(&s.place[bin_of(v)], 1u) - 1u] = v;
        }
        // (a bin's place now is where it begins, and that of the bin behind it where it ends)
      }
      int per = 1;   // threads to a token
      while (2 * per * m <= NT && per < 64) per *= 2;
      const int t = tid / per, sub = tid & (per - 1);
      __syncthreads();
      int lo = 0, many = t < m ? m : 0;
      u64 mine = 0;
      if (t < m) {
        mine = from[t];
        if (together) {
          const int b = bin_of(mine);
          lo = (int)s.place[b];
          many = (b + 1 < BINS ? (int)s.place[b + 1] : m) - lo;
          lo = lo & ~1, many += (int)s.place[b] & 1;   // (from an even place on: the one ahead of the bin's is less)
        }
      }
      const int len = ((many + per - 1) / per + 7) / 8 * 8;   // (what lies behind a bin's tokens is not less than they are)
      int ahead = less(from + lo + sub * len, len, mine);
      for (int d = 1; d < per; d <<= 1) ahead += __shfl_xor(ahead, d);
      __syncthreads();
      if (t < m && sub == 0) s.list[lo + ahead] = mine;
      __syncthreads();
    } else {
      for (int i = tid; i < CAP; i += NT) s.list[i] = i < m ? s.run[i] : ~0ull;
      int size = 256;
      while (size < m) size *= 2;
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
      __syncthreads();
    }
    for (int i = tid; i < (m <= NT ? NT : CAP); i += NT) {
      u64 w = 0;
      if (i < m) {
        const float l = listed(i);
        w = weight(l);
        if (masses) {
          const int b = bin(distance(l)), before = i ? bin_of(s.list[i - 1]) : -1;
          if (b != before) w += (b ? s.mass[b - 1] : 0) - (before >= 0 ? s.mass[before] : 0);
        }
      }
      s.run[i] = w;
    }
    __syncthreads();
    u64 total;
    if (m <= NT) running<NT>(s.run, s.wave64, &total);
    else running<CAP>(s.run, s.wave64, &total);
  }

  // ---- which bins hold the places that matter, s.count and s.mass being running sums.  `have_masses`: not, where top_k tokens are to be listed from the first on.
  __device__ __forceinline__ void plan(const Settings& t, bool have_masses, unsigned tokens, u64 total) {
    const bool cut_k = t.top_k && (unsigned)t.top_k <= tokens;
    const int bk = cut_k ? first_of<false>(s.count, BINS, (unsigned)t.top_k) : BINS - 1;
    const bool here = have_masses && cut_k;
    // the kept tokens' mass lies between these (the token where top-k cuts may weigh nothing)
    u64 lo = here ? max(bk ? s.mass[bk - 1] : 0, (u64)1) : total, hi = here ? s.mass[bk] : total;
    int p0 = BINS, p1 = BINS, m0 = BINS, m1 = BINS, u0 = BINS, u1 = BINS;   // (no bin)
    if (have_masses && t.cut_p) {
      lo = max(part_up(t.top_p, lo), (u64)1);
      hi = max(part_up(t.top_p, hi), (u64)1);
      p0 = first_of<false>(s.mass, BINS, lo);
      p1 = first_of<false>(s.mass, BINS, hi);
      hi = s.mass[p1];
    }
    if (have_masses && t.cut_min) {   // (a token's bin and its weight are rounded apart from each other: a bin more on either side)
      const int m = min((int)fmin(-0.5 * t.z_min / per_unit * (double)to_bin, (double)BINS), BINS - 1);
      m0 = max(m - 1, 0);
      m1 = min(m + 1, BINS - 1);
      lo = min(lo, max(m > 1 ? s.mass[m - 2] : 0, (u64)1));
      hi = min(hi, s.mass[m1]);
    }
    if (have_masses) {
      u0 = first_of<true>(s.mass, BINS, part_of(t.u, lo));
      u1 = first_of<true>(s.mass, BINS, part_of(t.u, hi));
    }
    static_assert(BINS == 4 * NT, "a thread's bins");
    of_k.first = here ? bk : have_masses ? BINS : 0;
    of_k.last = here || !have_masses ? bk : BINS;
    of_p.first = p0, of_p.last = p1;
    of_min.first = m0, of_min.last = m1;
    of_u.first = u0, of_u.last = u1;
    unsigned flags = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) flags |= wanted(tid * 4 + i) ? 1u << (8 * i) : 0u;
    reinterpret_cast<unsigned*>(s.gathered)[tid] = flags;
    __syncthreads();
  }

  // ---- the bins that hold the first top_k tokens, from the maxima of parts of the row (`have` of them, one to a thread, s.count being zero); false: not known
  __device__ __forceinline__ bool plan_by_maxima(const Settings& t, float maximum, bool have) {
    const float d = distance(maximum);
    if (have && weighs(d)) atomicAdd(&s.count[bin(d)], 1u);
    __syncthreads();
    unsigned tokens;
    running<BINS>(s.count, s.wave32, &tokens);
    plan(t, false, tokens, 0);
    return tokens >= (unsigned)t.top_k;
  }

  // ---- the token, from the sorted list of m tokens and the bins
  __device__ __forceinline__ int choose(const Settings& t, bool bins, unsigned tokens, u64 total, int m, u64* kept_mass) const {
    u64 kept = bins ? total : s.run[m - 1];
    if (t.top_k && (!bins || (unsigned)t.top_k < tokens)) {
      int rank = t.top_k - 1;   // its place in the list
      if (bins) {
        const int b = first_of<false>(s.count, BINS, (unsigned)t.top_k);
        rank -= (int)(b ? s.count[b - 1] : 0);
        for (int i = tid; i < m; i += NT)
          if (bin(distance(listed(i))) == b && (i == 0 || bin(distance(listed(i - 1))) != b)) s.found = i;
        __syncthreads();
        rank += s.found;
        __syncthreads();
      }
      kept = s.run[min(rank, m - 1)];
    }
    if (t.cut_p) kept = s.run[first_of<false>(s.run, m, max(part_up(t.top_p, kept), (u64)1))];
    if (t.cut_min) {   // (the first of all always stays)
      if (tid == 0) s.found = -1;
      __syncthreads();
      for (int i = tid; i < m; i += NT)
        if (exponent(listed(i)) >= t.z_min && (i + 1 == m || !(exponent(listed(i + 1)) >= t.z_min))) s.found = i;
      __syncthreads();
      u64 least = s.found >= 0 ? s.run[s.found] : 0;
      __syncthreads();
      if (bins && of_min.first > 0) least = max(least, s.mass[of_min.first - 1]);
      kept = min(kept, least);
    }
    *kept_mass = kept;
    return first_of<true>(s.run, m, part_of(t.u, kept));
  }

  // ---- where a bin's tokens do not fit the list: place by place, a crowded bin's tokens told apart by the digits of their keys
  enum Goal { RANK, REACH, PASS };
  struct Place { u64 mass; int number; float logit; };   // of the tokens up to the place, with its own; the token there (PASS)
  __device__ __forceinline__ Place within(int b, Goal kind, u64 goal) const {
    unsigned prefix = 0;
    int shift = 32;
    u64 base = 0;
    __syncthreads();   // (the next gathering clears s.listed, which a late wave may still be reading behind the one before)
    for (;;) {
      vec first[2];
      load(first, piece0 + tid);
      auto here = [&](float l) {
        const float d = distance(l);
        return weighs(d) && bin(d) == b && (shift == 32 || key_of(l) >> shift == prefix);
      };
      const int m = gather(here, here, first);
      if (m <= CAP) {
        sort(m, false);
        const int i = kind == RANK ? (int)goal - 1 : kind == REACH ? first_of<false>(s.run, m, goal) : first_of<true>(s.run, m, goal);
        return {base + s.run[i], number(i), listed(i)};
      }
      if (shift == 0) break;
      const int digits = shift == 10 ? 10 : 11, next = shift - digits, mask = (1 << digits) - 1;
      __syncthreads();
      for (int i = tid; i < BINS; i += NT) s.count2[i] = 0, s.mass2[i] = 0;
      __syncthreads();
      each<1>([&](float l, int) {
        const float d = distance(l);
        const unsigned key = key_of(l);
        if (weighs(d) && bin(d) == b && (shift == 32 || key >> shift == prefix)) {
          const int digit = mask - (int)(key >> next & (unsigned)mask);   // (descending)
          atomicAdd(&s.count2[digit], 1u);
          atomicAdd(&s.mass2[digit], weight(l));
        }
      });
      __syncthreads();
      unsigned tc;
      u64 tm;
      running<BINS>(s.count2, s.wave32, &tc);
      running<BINS>(s.mass2, s.wave64, &tm);
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
      for (int i = lo; i < hi; ++i) mine += key_of((float)logits[i]) == prefix;
      const unsigned end = scan<unsigned>(mine, s.wave32, &total);
      if (end >= which && end - mine < which) {
        unsigned at = end - mine;
        for (int i = lo; i < hi; ++i)
          if (key_of((float)logits[i]) == prefix && ++at == which) s.found = i;
      }
      __syncthreads();
      num = s.found;
      __syncthreads();
    }
    return {base + which * w, num, l};
  }
  // a place among all tokens, from the bins' running sums
  __device__ __forceinline__ Place among(Goal kind, u64 goal) const {
    const int b = kind == RANK ? first_of<false>(s.count, BINS, (unsigned)goal)
                               : kind == REACH ? first_of<false>(s.mass, BINS, goal) : first_of<true>(s.mass, BINS, goal);
    const u64 ahead = b ? s.mass[b - 1] : 0;
    Place p = within(b, kind, goal - (kind == RANK ? (u64)(b ? s.count[b - 1] : 0) : ahead));
    p.mass += ahead;
    return p;
  }
  __device__ __forceinline__ Place by_places(const Settings& t, unsigned tokens, u64 total, u64* kept_mass) const {
    u64 kept = total;
    Place place{0, 0, top};
    for (int step = 0; step < 4; ++step) {
      if ((step == 0 && !(t.top_k && (unsigned)t.top_k < tokens)) || (step == 1 && !t.cut_p) || (step == 2 && !t.cut_min)) continue;
      if (step == 2) {
        u64 mine = 0, sum;
        each<1>([&](float l, int) { if (weighs(distance(l)) && exponent(l) >= t.z_min) mine += weight(l); });
        scan<u64>(mine, s.wave64, &sum);
        kept = min(kept, sum);
        continue;
      }
      place = among(step == 0 ? RANK : step == 1 ? REACH : PASS,
                    step == 0 ? (u64)t.top_k : step == 1 ? max(part_up(t.top_p, kept), (u64)1) : part_of(t.u, kept));
      if (step < 3) kept = place.mass;
    }
    *kept_mass = kept;
    return place;
  }

  // ---- a whole row.  ready: s.count and s.mass hold the bins of all of it, s.run its list of m tokens or, m > CAP, nothing.
  __device__ __forceinline__ void finish(const SampleArgs& a, int r, const Settings& t, bool ready, int m) {
    bool bins = false, masses = t.masses();
    unsigned tokens = 0;
    u64 total = 0, kept = 0;
    int token = 0;
    float logit = top;
    bool by_value = t.by_value(), by_maxima = !ready && t.by_maxima(NT);
    for (;;) {
      bool known = true;
      if (by_maxima) {
        clear_bins();
        known = plan_by_maxima(t, own, true);
      } else if (!by_value && !ready) {
        clear_bins();
        fill_bins(t.top_k, masses);
        running<BINS>(s.count, s.wave32, &tokens);
        running<BINS>(s.mass, s.wave64, &total);
        plan(t, masses, tokens, total);
      } else if (!by_value) {
        tokens = s.count[BINS - 1];
        total = s.mass[BINS - 1];
      }
      if (!known) m = CAP + 1;
      else if (!ready) {
        vec first[2];
        load(first, piece0 + tid);
        m = by_value ? gather_value(t.z_min, first) : gather_bins(first);
      }
      bins = !by_value && !by_maxima && masses;
      if (m <= CAP || bins) break;
      masses = masses || !by_maxima;   // (without the maxima first by counts alone, if that may do)
      by_value = by_maxima = ready = false;
    }
    if (m <= CAP) {
      sort(m, bins);
      const int i = choose(t, bins, tokens, total, m, &kept);
      token = number(i);
      logit = listed(i);
    } else {
      const Place p = by_places(t, tokens, total, &kept);
      token = p.number;
      logit = p.logit;
    }
    if (tid == 0) {
      a.tokens[r] = token;
      if (a.probs) a.probs[r] = (float)(pow2(exponent(logit)) / ldexp((double)kept, -scale_bits));
    }
  }
};

__device__ __forceinline__ void leave_first(const SampleArgs& a, int r, const Top& t) {
  const bool any = t.best > -__builtin_inff();
  a.tokens[r] = any ? t.at : -1;
  if (a.probs) a.probs[r] = any ? 1.f : 0.f;
}

// a workgroup to a row
template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(const SampleArgs a) {
  __shared__ Lds s;
  const int r = (int)blockIdx.x;
  Row<T> row(s, a, r);
  const Settings t(a, r);
  const Top top = row.extremes(t);
  if (top.best == -__builtin_inff() || t.greedy) {
    if (threadIdx.x == 0) leave_first(a, r, top);
    return;
  }
  row.set(top, t.temperature);
  row.finish(a, r, t, false, 0);
}

// What the workgroups of a row leave each other.  The first launch clears what the others add to.
struct Shared {
  u64 mass[BINS];
  u64 list[CAP];
  unsigned count[BINS];
  Top top[PARTS];
  float maxima[PARTS * WAVES];   // of what a wave has read
  unsigned listed, arrived;
  unsigned pad[14];
};

template <typename T>
__global__ __launch_bounds__(NT) void sample_top_kernel(const SampleArgs a) {
  __shared__ Lds s;
  const int g = (int)blockIdx.x, parts = (int)gridDim.x, r = (int)blockIdx.y;
  Shared& h = static_cast<Shared*>(a.workspace)[r];
  Row<T> row(s, a, r);
  row.share(g, parts);
  const Top t = row.extremes(Settings(a, r));
  if (threadIdx.x == 0) {
    h.top[g] = t;
    if (g == 0) h.listed = h.arrived = 0;
  }
  const float most = wave_fold32(row.own, [](float x, float y) { return fmaxf(x, y); });
  if ((threadIdx.x & 63) == 0) h.maxima[g * WAVES + (threadIdx.x >> 6)] = most;
  for (int i = BINS * g / parts + (int)threadIdx.x; i < BINS * (g + 1) / parts; i += NT) h.mass[i] = 0, h.count[i] = 0;
}

__device__ __forceinline__ Top top_of(const Shared& h, int parts) {
  Top t{-__builtin_inff(), __builtin_inff(), 0x7fffffff};
  const int lane = (int)threadIdx.x & 63;
  if (lane < parts) t = h.top[lane];
  return of_wave(t);
}

template <typename T>
__global__ __launch_bounds__(NT) void sample_bins_kernel(const SampleArgs a) {
  __shared__ Lds s;
  const int r = (int)blockIdx.y;
  Shared& h = static_cast<Shared*>(a.workspace)[r];
  Row<T> row(s, a, r);
  const Settings t(a, r);
  row.share((int)blockIdx.x, (int)gridDim.x);
  typename Row<T>::vec first[1];   // (on its way while the maximum is looked up)
  row.load(first, row.piece0 + row.tid);
  const Top top = top_of(h, (int)gridDim.x);
  if (top.best == -__builtin_inff() || t.greedy || t.by_value() || t.by_maxima((int)gridDim.x * WAVES)) return;
  row.set(top, t.temperature);
  row.clear_bins();
  row.fill_bins(t.top_k, t.masses(), first);
  for (int i = (int)threadIdx.x; i < BINS; i += NT) {
    if (s.count[i]) atomicAdd(&h.count[i], s.count[i]);
    if (s.mass[i]) atomicAdd(&h.mass[i], s.mass[i]);
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void sample_pick_kernel(const SampleArgs a) {
  __shared__ Lds s;
  const int r = (int)blockIdx.y, tid = (int)threadIdx.x;
  Shared& h = static_cast<Shared*>(a.workspace)[r];
  Row<T> row(s, a, r);
  const Settings t(a, r);
  row.share((int)blockIdx.x, (int)gridDim.x);
  typename Row<T>::vec first[2];   // (on its way while the bins are looked through)
  row.load(first, row.piece0 + tid);
  static_assert(PARTS * WAVES <= NT, "a maximum to a thread");
  const int maxima = (int)gridDim.x * WAVES;
  const float maximum = tid < maxima ? h.maxima[tid] : 0.f;
  unsigned count[BINS / NT];
  u64 mass[BINS / NT];
#pragma unroll
  for (int i = 0; i < BINS / NT; ++i) count[i] = h.count[i * NT + tid], mass[i] = h.mass[i * NT + tid];
  const Top top = top_of(h, (int)gridDim.x);
  if (top.best == -__builtin_inff() || t.greedy) {
    if (blockIdx.x == 0 && tid == 0) leave_first(a, r, top);
    return;
  }
  row.set(top, t.temperature);
  const bool by_value = t.by_value(), by_maxima = t.by_maxima(maxima);
  bool known = true;
  if (by_maxima) {
    row.clear_bins();
    known = row.plan_by_maxima(t, maximum, tid < maxima);
  } else if (!by_value) {
#pragma unroll
    for (int i = 0; i < BINS / NT; ++i) s.count[i * NT + tid] = count[i], s.mass[i * NT + tid] = mass[i];
    __syncthreads();
    unsigned tokens;
    u64 total;
    row.template running<BINS>(s.count, s.wave32, &tokens);
    row.template running<BINS>(s.mass, s.wave64, &total);
    row.plan(t, t.masses(), tokens, total);
  }
  const int m = !known ? CAP + 1 : by_value ? row.gather_value(t.z_min, first) : row.gather_bins(first);
  // this part's tokens to the row's list (in any order: it is sorted), and whoever is last ends the row
  if (tid == 0) s.found = (int)min(__hip_atomic_fetch_add(&h.listed, (unsigned)m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), 1u << 30);
  __syncthreads();
  const int base = s.found;
  if (m <= CAP)
    for (int i = tid; i < m && base + i < CAP; i += NT) __hip_atomic_store(&h.list[base + i], s.run[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s.found = __hip_atomic_fetch_add(&h.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  __syncthreads();
  if (!s.found) return;
  const int all = (int)min(__hip_atomic_load(&h.listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), (unsigned)CAP + 1);
  __syncthreads();
  if (all <= CAP)
    for (int i = tid; i < all; i += NT) s.run[i] = __hip_atomic_load(&h.list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  row.share(0, 1);
  row.finish(a, r, t, true, all);
}

template <typename T>
hipError_t launch_type(const SampleArgs& a, int parts, hipStream_t st) {
  if (!a.workspace || parts == 1) {
    constexpr int kMost = 1 << 22;   // rows of a launch: one has fewer than 2^32 threads
    for (long first = 0; first < a.rows; first += kMost) {
      SampleArgs b = a;
      b.rows = (int)(a.rows - first < kMost ? a.rows - first : kMost);
      b.logits = static_cast<const T*>(a.logits) + first * a.logits_stride;
      auto on = [&](auto*& p) { if (p) p += first; };
      on(b.temperature), on(b.top_k), on(b.top_p), on(b.min_p), on(b.uniform), on(b.tokens), on(b.probs);
      hipLaunchKernelGGL((sample_kernel<T>), dim3((unsigned)b.rows), dim3(NT), 0, st, b);
      if (hipError_t e = hipGetLastError()) return e;
    }
  } else {
    const dim3 grid((unsigned)parts, (unsigned)a.rows), block(NT);
    hipLaunchKernelGGL((sample_top_kernel<T>), grid, block, 0, st, a);
    hipLaunchKernelGGL((sample_bins_kernel<T>), grid, block, 0, st, a);
    hipLaunchKernelGGL((sample_pick_kernel<T>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

// A row to a workgroup, or to as many as give every CU one.  Measured in graphs, bf16, us in one launch / shared out, top-p 0.9 alone and top-k 50 with top-p 0.95: one row of 16000 tokens 17 / 20 and 11 / 26,
// of 32000 23 / 21 and 13 / 17, of 64000 37 / 21 and 17 / 17, of 128000 63 / 23 and 23 / 17; 64 rows of 32000 26 / 26 and 14 / 23, of 64000 42 / 32 and 18 / 25, of 128000 81 / 51 and 26 / 30; 128 rows of 64000
// 44 / 41 and 19 / 31, of 128000 84 / 68 and 29 / 41.  256 rows of 50257 in fp32, each with its own settings, 49 / 54 (two to a row).  What a row is asked for is known on the device alone: where there may be
// top-k rows must be longer.
int parts_of(const SampleArgs& a) {
  const int parts = a.rows >= 256 ? 1 : 256 / a.rows < 32 ? 256 / a.rows : 32;
  return (long)a.vocab * (parts - 1) >= (a.top_k ? 36000L : 24000L) * parts ? parts : 1;
}

}  // namespace

size_t sample_workspace_need(const SampleArgs& a) { return parts_of(a) > 1 ? (size_t)a.rows * sizeof(Shared) : 0; }
size_t sample_workspace_bytes(const SampleArgs& a) {
  SampleArgs b = a;
  for (b.rows = a.rows < 128 ? a.rows : 128; b.rows > 0; b.rows = 256 / (256 / b.rows + 1))   // (the most rows that have a share more each; more than 128 have one)
    if (parts_of(b) > 1) return sample_workspace_need(b);
  return 0;
}

hipError_t launch_sample(const SampleArgs& args, int dtype, hipStream_t st) {
  SampleArgs a = args;
  int bits = 0;   // vocab <= 2^bits
  while ((1 << bits) < a.vocab) ++bits;
  a.scale_bits = 62 - bits < 51 ? 62 - bits : 51;
  const int parts = parts_of(a);
  if (dtype == T_F16) return launch_type<_Float16>(a, parts, st);
  return dtype == T_BF16 ? launch_type<__bf16>(a, parts, st) : launch_type<float>(a, parts, st);
}

}  // namespace relay
