// Sampling from rows of logits, from given random numbers.
//
//   tokens in order of their logits, equal ones by index; e_j = e^(scale (z_j -
//   z_0)). Kept are the first of them: top_k at most; then those before which
//   less than top_p of the mass lies; of these, the ones with e_j >= min_p.
//   The token: the first in that order with e_0 + .. + e_j > r sum of the kept.
//
// Filters and the draw are then one question asked up to four times: at which
// token of the order does a count, or a running mass, pass a bound? Nothing is
// sorted. A row's tokens are counted into bins of 1/32 nat below its maximum,
// with their mass; the bin that the bound falls into is cut again by the bits
// of the logits until one value is left, whose tokens are equal. Masses are
// fixed-point sums relative to their bin's middle (2^-42 of it, 64 bits): exact,
// and the same in whatever order the atomics come.
//   Rows of 16 bits that fit a workgroup's registers go another way, below.
//
//   Where few tokens may be kept (top_k of 1024 and less, min_p alone), what
// lies below a bound for them is not counted, and up to 256 that are left are
// ordered at once.
//
// Neither is bound by memory: a row is one workgroup's work, on one CU. Of fp32
// 126464 logits take 18 to 20 us with top_k 40, 44 without a filter, 48 with
// top_p; 128 such rows 28, 58 to 68 and 62, 7 rows of 32003 with min_p 13 to 15.
// What takes the time is an LDS addition of 64 bits (four times one of 32) and
// an exponential for each token that is counted, and the steps between the
// workgroup's barriers. Flat rows (0.05 N(0, 1)), whose tokens meet in few bins,
// take 120 without a filter and 165 with top_p, 128 of them 130 and 183.
#include <cstdint>

#include "logit_rows.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2 * kThreads, kFar = kBins - 1;   // the last bin: e^-63.97 and less, of no mass
constexpr double kPerNat = 32.0;
constexpr double kUnit = 4398046511104.0;   // 2^42

// order of floats as unsigned numbers (a negative zero is made positive before)
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}

// Bin and mass of a logit. The bin is the nearest one in float32 (it falls as
// the logit rises, which is all that is asked of it); the mass relative to the
// bin's middle, e^x with x the distance from there, is of float64: its series
// to the fourth power, the fifth spread over the others as Chebyshev
// polynomials are (x^5 = 5/4 h^2 x^3 - 5/16 h^4 x to within h^5 / 16 for |x| <=
// h = 1/64: 5e-13 of the mass).
// The bin is taken of half the distance, since the whole one may be beyond float32: 3e38 and -1e38 at a scale of 1e-38 are
// 4 nats apart. Halving is exact but for subnormals, whose lost bit is 2^-44 of a bin at the largest scale.
struct Weigh {
  float top, half, k;   // maximum, half of it, bins per unit of logit
  double m, scale;
  __device__ __forceinline__ Weigh(float t, float s)
      : top(t), half(0.5f * t), k(s * (float)kPerNat), m((double)t), scale((double)s) {}
  // nats below the maximum
  __device__ __forceinline__ double below(float z) const { return (m - (double)z) * scale; }
  __device__ __forceinline__ float bin_of(float z) const { return rintf(fminf(fmaf(-0.5f, z, half) * (2.f * k), (float)kFar)); }
  __device__ __forceinline__ int bin(float z) const { return (int)bin_of(z); }
  // fixed-point mass of a logit in bin b
  __device__ __forceinline__ unsigned long long mass(float z, float b) const {
    const double x = fma((double)z - m, scale, (double)(b * (float)(1.0 / kPerNat)));   // |x| about 1/64 at most
    constexpr double h2 = 1.0 / 4096;
    double p = fma(x, 1.0 / 24, 1.0 / 6 + 1.25 / 120 * h2);
    p = fma(x, p, 0.5);
    p = fma(x, p, 1.0 - 0.3125 / 120 * h2 * h2);
    p = fma(x, p, 1.0);
    // 2^52 added: the integer nearest to p 2^42 is the sum's low bits
    return (unsigned long long)__double_as_longlong(fma(p, kUnit, 4503599627370496.0)) & 0xfffffffffffffull;
  }
  // what a bin's fixed-point masses are worth: nothing in the last one
  static __device__ __forceinline__ double unit(int b) { return b == kFar ? 0.0 : exp(-(double)b / kPerNat) / kUnit; }
};

// inclusive sums over a wave's lanes, by moves between neighbouring registers' lanes (a shuffle through LDS takes ten
// times as long, and these stand in a chain)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lanes_below(uint32_t v) {   // of the lane that CTRL names, 0 where there is none
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double lanes_below(double v) {
  return __hiloint2double((int)lanes_below<CTRL, ROWS>((uint32_t)__double2hiint(v)),
                          (int)lanes_below<CTRL, ROWS>((uint32_t)__double2loint(v)));
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
  v += lanes_below<0x111, 0xf>(v);   // 1, 2, 4, 8 lanes below in a row of 16
  v += lanes_below<0x112, 0xf>(v);
  v += lanes_below<0x114, 0xf>(v);
  v += lanes_below<0x118, 0xf>(v);
  v += lanes_below<0x142, 0xa>(v);   // the last lane of the row below, into rows 1 and 3
  v += lanes_below<0x143, 0xc>(v);   // lane 31, into rows 2 and 3
  return v;
}
__device__ __forceinline__ double lane_of(double v, int at) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), at), __builtin_amdgcn_readlane(__double2loint(v), at));
}

// All that may be kept, where it is few: no bins, but the tokens in their order, each thread counting those before its own.
// One row of 126464 with top_k 40 and top_p takes 16.4 us so and 20.4 by the table of 16-bit values, 17.6 and 34.7 by bins;
// with more tokens than these the counting, which grows with their square, takes as long as the bins.
constexpr int kShort = 256;
struct Short {
  unsigned long long key[kShort];   // places in the order, without their ties
  double e[kShort];                 // masses in that order
  int index[kShort];
  uint32_t in[kShort / 64], kept;
};
struct Filters {
  int top_k;
  float top_p, r;
  bool least;
  double limit;
};
// Of thread t the t-th of `seen` tokens, of place `slot` (rising in the order) and `index`; `all` may be kept before top_k.
// Writes the row's token, prob and kept; returns the tokens kept, and the thread's rank.
__device__ __forceinline__ uint32_t draw_short(Short& s, const SampleCall& a, int n, const Weigh& w, const Filters& f,
                                               uint32_t seen, uint32_t all, uint32_t slot, int index, float z, uint32_t& rank) {
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6;
  const bool mine = t < (int)seen;
  const unsigned long long key = mine ? (unsigned long long)slot << 32 | (uint32_t)index : ~0ull;
  if (t < kShort) {
    s.key[t] = key;
    if (!mine) s.e[t] = 0.0;
  }
  __syncthreads();
  rank = 0;
  if (t < kShort) {
    if (wid * 64 < (int)seen) {
#pragma unroll 8
      for (int k = 0; k < ((int)seen + 7) / 8 * 8; ++k) rank += s.key[k] < key;
    }
    const double below = w.below(z);
    if (mine) {
      s.e[rank] = exp(-below);
      s.index[rank] = index;
    }
    const unsigned long long in = __ballot(mine && below <= f.limit);
    if (lane == 0) s.in[wid] = __popcll(in);
  }
  __syncthreads();
  if (wid == 0) {   // four tokens a lane
    double e[4], m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = s.e[4 * lane + i];
    const double own = (e[0] + e[1]) + (e[2] + e[3]), upto = wave_scan(own);
    m[0] = (upto - own) + e[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) m[i] = m[i - 1] + e[i];
    auto of = [&](const double (&x)[4], uint32_t i) {
      const uint32_t c = i & 3;
      return lane_of(c == 0 ? x[0] : c == 1 ? x[1] : c == 2 ? x[2] : x[3], i >> 2);
    };
    // of the first `among`, how many hold
    auto count = [&](uint32_t among, auto holds) {
      uint32_t c = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c += __popcll(__ballot(4 * lane + i < (int)among && holds(m[i])));
      return c;
    };
    uint32_t kept = all;
    if (f.top_k > 0) kept = min(kept, (uint32_t)f.top_k);
    double mass = of(m, kept - 1);
    if (f.top_p < 1.f) {
      const double bound = fmax((double)f.top_p, 0.0) * mass;
      kept = min(kept, 1 + count(kept, [&](double x) { return x < bound; }));
    }
    if (f.least) {
      uint32_t in = 0;
#pragma unroll
      for (int i = 0; i < kShort / 64; ++i) in += s.in[i];
      kept = min(kept, in);
    }
    kept = __builtin_amdgcn_readfirstlane(kept);
    mass = of(m, kept - 1);
    const double bound = fmin(fmax((double)f.r, 0.0), 1.0) * mass;
    const uint32_t at = __builtin_amdgcn_readfirstlane(min(kept - 1, count(kept, [&](double x) { return x <= bound; })));
    const double p = of(e, at);
    if (lane == 0) {
      a.token[n] = s.index[at];
      if (a.prob) a.prob[n] = (float)(p / mass);
      if (a.kept) a.kept[n] = (int)kept;
      s.kept = kept;
    }
  }
  __syncthreads();
  return s.kept;
}
// whether it can: what top_k keeps has been seen
__device__ __forceinline__ bool short_enough(uint32_t seen, uint32_t all, int top_k) {
  return seen <= kShort && (top_k <= 0 || ((uint32_t)top_k < all ? (uint32_t)top_k <= seen : seen == all));
}

// The token found: the `at`-th (by index) of `eq` tokens of the logit `key`, before which lie n tokens of mass m; each has
// mass w.
struct Place {
  uint32_t key, n, eq, at;
  int index;   // or -1: not known yet
  double m, w;
  __device__ __forceinline__ uint32_t rank() const { return n + at; }
  __device__ __forceinline__ double upto() const { return m + (double)(at + 1) * w; }
};

// Where a bound falls among the bins, with what lies before it: n tokens of mass m before the bin of `count`.
struct Spot {
  int bin;
  uint32_t n, count;
  double m;
};
struct Counts {
  uint32_t n[kBins];   // tokens
  unsigned long long mass[kBins];
};
struct Bins : Counts {
  uint32_t n_upto[kBins];   // and up to the bin's end
  double m_upto[kBins];
};

constexpr int kListed = 4096;   // tokens of a bin that are taken out of the row

struct Shared {
  union {
    struct {
      Bins all, part;
    };
    Short few;
    Counts copies[4];   // a row's tokens are counted by every fourth lane apart: half of a wave would meet in one place
  };
  uint32_t list_key[kListed];      // the tokens with keys list_lo .. list_hi (an empty range at first)
  int list_index[kListed];
  uint32_t listed, list_lo, list_hi;
  uint32_t from;                   // keys below are not counted
  uint32_t few_key[64];            // a bin's tokens, where they are few
  int few_index[64];
  uint32_t wave_n[kWaves];
  double wave_m[kWaves];
  float wave_top[kWaves];
  int wave_bad[kWaves];
  uint32_t wave_in[kWaves];
  uint32_t lo, hi;
  Spot spot;
  int token;
  uint32_t slab[64];
  Place place;
};

// f(values, their number, index) of the row's entries: eight at a time, and at last one
template <class E, class F>
__device__ __forceinline__ void each_eight(const typename E::t* row, int V, F f) {
  constexpr int kFlight = 4;
  const int whole = V & ~7;
  for (int i0 = 8 * threadIdx.x; i0 < whole; i0 += kFlight * 8 * kThreads) {
    Eight<E> v[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (i0 + u * 8 * kThreads < whole) v[u].load(row + i0 + u * 8 * kThreads);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int i = i0 + u * 8 * kThreads;
      if (i < whole) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = v[u].at(e);
        f(z, i);
      }
    }
  }
  const int i = whole + threadIdx.x;
  if (i < V) {
    const float z[1] = {E::one(row + i)};
    f(z, i);
  }
}
// f(value, index), a negative zero made positive
template <class E, class F>
__device__ __forceinline__ void each(const typename E::t* row, int V, F f) {
  each_eight<E>(row, V, [&](auto& z, int i) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(z) / sizeof(float)); ++e) f(z[e] + 0.f, i + e);
  });
}
// the largest of some values (NaN if there is one), three at a time
template <int N>
__device__ __forceinline__ float largest(float top, const float (&z)[N]) {
#pragma unroll
  for (int e = 0; e + 1 < N; e += 2) top = __builtin_elementwise_maximum(top, __builtin_elementwise_maximum(z[e], z[e + 1]));
  return N == 1 ? __builtin_elementwise_maximum(top, z[0]) : top;
}
template <int N>
__device__ __forceinline__ float smallest(const float (&z)[N]) {
  float low = z[0];
#pragma unroll
  for (int e = 1; e < N; ++e) low = __builtin_elementwise_minimum(low, z[e]);
  return low;
}

__device__ __forceinline__ void clear(Bins& b) {
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    b.n[i] = 0;
    b.mass[i] = 0;
  }
}

// running counts and masses over the bins, two a thread; unit: of a bin's mass, or one for all
template <bool COARSE>
__device__ __forceinline__ void scan(Bins& b, double unit, Shared& s) {
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6;
  uint32_t n[2];
  double m[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    n[j] = b.n[2 * t + j];
    m[j] = (double)b.mass[2 * t + j] * (COARSE ? Weigh::unit(2 * t + j) : unit);
  }
  const uint32_t sn = wave_scan(n[0] + n[1]);
  const double sm = wave_scan(m[0] + m[1]);
  if (lane == 63) {
    s.wave_n[wid] = sn;
    s.wave_m[wid] = sm;
  }
  __syncthreads();
  uint32_t bn = 0;
  double bm = 0.0;
  for (int w = 0; w < wid; ++w) {
    bn += s.wave_n[w];
    bm += s.wave_m[w];
  }
  b.n_upto[2 * t + 1] = bn + sn;
  b.m_upto[2 * t + 1] = bm + sm;
  b.n_upto[2 * t] = bn + sn - n[1];
  b.m_upto[2 * t] = bm + (sm - m[1]);
  __syncthreads();
}

// A bound in the order of the tokens: the token of a rank, or the first one whose running mass passes (or reaches) a mass.
struct Bound {
  bool by_rank, reach;
  uint32_t rank;
  double mass;
};
// By the first wave: the first of its lanes in whose running sums the bound is passed (by rounding alone, the last that
// holds anything).
__device__ __forceinline__ int first_of(const Bound& q, uint32_t n, double m, uint32_t before, bool in) {
  const bool some = in && n > before;
  const bool past = q.by_rank ? n > q.rank : q.reach ? m >= q.mass : m > q.mass;
  const unsigned long long hits = __ballot(some && past), any = __ballot(some);
  return hits ? __builtin_ctzll(hits) : any ? 63 - __builtin_clzll(any) : 0;
}

// of eq equal tokens of mass w each, which follow n tokens of mass m, the one at which the bound is passed
__device__ __forceinline__ uint32_t which_of(const Bound& q, uint32_t n, double m, double w, uint32_t eq) {
  if (q.by_rank) return min(q.rank - n, eq - 1);
  if (eq == 1) return 0;
  auto past = [&](double i) { return q.reach ? m + (i + 1.0) * w >= q.mass : m + (i + 1.0) * w > q.mass; };
  double i = w > 0.0 ? floor((q.mass - m) / w) : 0.0;
  i = fmin(fmax(i, 0.0), (double)(eq - 1));
  while (i > 0.0 && past(i - 1.0)) i -= 1.0;
  while (i < (double)(eq - 1) && !past(i)) i += 1.0;
  return (uint32_t)i;
}

// by the first wave: of 32 times 64 bins, whose sums follow n0 tokens of mass m0
__device__ __forceinline__ Spot locate(const Bins& b, const Bound& q, uint32_t n0, double m0) {
  const int lane = threadIdx.x & 63, g = (lane & 31) * 64;
  const int group = first_of(q, n0 + b.n_upto[g + 63], m0 + b.m_upto[g + 63], n0 + (g ? b.n_upto[g - 1] : 0), lane < 32);
  const int i = group * 64 + lane;
  const int bin = group * 64 + first_of(q, n0 + b.n_upto[i], m0 + b.m_upto[i], n0 + b.n_upto[i] - b.n[i], true);
  const uint32_t before = b.n_upto[bin] - b.n[bin];
  return Spot{bin, n0 + before, b.n[bin], before == 0 ? m0 : m0 + b.m_upto[bin - 1]};
}

template <class E>
__device__ __forceinline__ Place find(const typename E::t* row, int V, const Weigh& w, uint32_t top, const Bound& q, Shared& s) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    const Spot p = locate(s.all, q, 0, 0.0);
    const int b = p.bin;
    // The bin's logits are an interval; its ends, 64 steps at once. The bin falls as the key rises: the largest key of a
    // bin >= b, then the smallest of a bin <= b.
    // It lies within 0.6 of its middle's place, a step of the floats around; where that place is beyond float32 or nearly,
    // anywhere.
    const uint32_t least = key_of(-3.402823466e38f);
    const float far = w.top - ((float)b + 0.6f) / w.k, near = w.top - ((float)b - 0.6f) / w.k;
    const uint32_t from = b == kFar || !(far > -3.0e38f) ? least : key_of(far) - 2;
    uint32_t lo = from, hi = b == 0 || !(near < w.top) || !(near > -3.0e38f) ? top : min(top, key_of(near) + 2);
    while (lo < hi) {   // bin(lo) >= b, the answer in lo .. hi
      const uint32_t step = (hi - lo) / 64 + 1;
      const uint32_t k = lo + (uint32_t)(lane + 1) * step;
      const int c = __popcll(__ballot(k <= hi && k > lo && w.bin(value_of(k)) >= b));   // the first c hold
      lo += c * step;
      hi = min(hi, lo + step - 1);
    }
    const uint32_t last = lo;
    lo = from;
    hi = last;
    while (lo < hi) {   // bin(hi) <= b
      const uint32_t step = (hi - lo) / 64 + 1;
      const uint32_t k = hi - (uint32_t)(lane + 1) * step;
      const int c = __popcll(__ballot(k >= lo && k < hi && w.bin(value_of(k)) <= b));
      hi -= c * step;
      lo = hi - lo >= step ? hi - step + 1 : lo;
    }
    if (lane == 0) {
      s.spot = p;
      s.lo = hi;
      s.hi = last;
    }
  }
  __syncthreads();
  const int b = s.spot.bin;
  uint32_t n = s.spot.n, count = s.spot.count;
  double m = s.spot.m;
  const double unit = Weigh::unit(b);
  uint32_t lo = max(s.lo, s.from), hi = s.hi;
  // a list of the bin's tokens, and of all before them where they fit as well (the next bound falls there)
  bool listed = s.list_lo <= lo && hi <= s.list_hi;
  if (!listed && count <= kListed) {
    const uint32_t to = s.all.n_upto[b] <= kListed ? top : hi;
    __syncthreads();
    if (threadIdx.x == 0) {
      s.listed = 0;
      s.list_lo = lo;
      s.list_hi = to;
    }
    __syncthreads();
    each<E>(row, V, [&](float z, int i) {
      const uint32_t k = key_of(z);
      if (k >= lo && k <= to) {
        const uint32_t at = atomicAdd(&s.listed, 1u);   // (as many as were counted)
        if (at < kListed) {
          s.list_key[at] = k;
          s.list_index[at] = i;
        }
      }
    });
    listed = true;
  }
  __syncthreads();
  if (listed && count <= 64) {   // by the first wave, a lane a token: each sees how many, and what mass, come before it
    if (threadIdx.x < 64) {
      uint32_t found = 0;
      for (uint32_t i0 = 0; i0 < s.listed; i0 += 64) {
        const uint32_t k = i0 + lane < s.listed ? s.list_key[i0 + lane] : 0;
        const bool mine = k >= lo && k <= hi;   // (lo > 0)
        const unsigned long long all = __ballot(mine);
        const uint32_t at = found + __popcll(all & ((1ull << lane) - 1ull));
        if (mine && at < 64) {
          s.few_key[at] = k;
          s.few_index[at] = s.list_index[i0 + lane];
        }
        found += __popcll(all);
      }
      __builtin_amdgcn_wave_barrier();
      const bool in = lane < (int)count;
      const uint32_t key = in ? s.few_key[lane] : 0;
      const int index = in ? s.few_index[lane] : 0;
      const unsigned long long units = in ? w.mass(value_of(key), (float)b) : 0;
      const double e = (double)units * unit;
      uint32_t above = 0, equal = 0, at = 0;
      unsigned long long over = 0;   // the mass above, whole units: the list has the order in which its places were taken
      for (int j = 0; j < (int)count; ++j) {
        const uint32_t kj = __builtin_amdgcn_readlane(key, j);
        const int ij = __builtin_amdgcn_readlane(index, j);
        const unsigned long long uj = (unsigned long long)__builtin_amdgcn_readlane((uint32_t)(units >> 32), j) << 32 |
                                      (uint32_t)__builtin_amdgcn_readlane((uint32_t)units, j);
        above += kj > key;
        over += kj > key ? uj : 0;
        equal += kj == key;
        at += kj == key && ij < index;
      }
      const double mass = m + (double)over * unit;
      const uint32_t order = above + at;
      const double upto = mass + (double)(at + 1) * e;
      const bool past = in && (q.by_rank ? n + order >= q.rank : q.reach ? upto >= q.mass : upto > q.mass);
      // the first that is past the bound, by rounding alone the last of all
      uint32_t best = past ? order : in ? 0x10000u + 64 - order : 0x20000u;
#pragma unroll
      for (int k = 32; k >= 1; k >>= 1) best = min(best, (uint32_t)__shfl_xor((int)best, k));
      if (in && best == (past ? order : 0x10000u + 64 - order)) s.place = Place{key, n + above, equal, at, index, mass, e};
    }
    __syncthreads();
    return s.place;
  }
  while (lo < hi) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __builtin_clz(span), shift = max(0, bits - 11);   // span >> shift < 2048
    __syncthreads();
    clear(s.part);
    __syncthreads();
    auto add = [&](uint32_t k) {
      if (k >= lo && k <= hi) {
        const int i = (int)((hi - k) >> shift);
        atomicAdd(&s.part.n[i], 1u);
        atomicAdd(&s.part.mass[i], w.mass(value_of(k), (float)b));
      }
    };
    if (listed) {
      for (uint32_t i = threadIdx.x; i < s.listed; i += kThreads) add(s.list_key[i]);
    } else {
      each<E>(row, V, [&](float z, int) { add(key_of(z)); });
    }
    __syncthreads();
    scan<false>(s.part, unit, s);
    if (threadIdx.x < 64) {
      const Spot p = locate(s.part, q, n, m);
      if (lane == 0) s.spot = p;
    }
    __syncthreads();
    const uint32_t i = s.spot.bin;
    n = s.spot.n;
    m = s.spot.m;
    count = s.spot.count;
    hi -= i << shift;
    const uint32_t width = (1u << shift) - 1;
    lo = hi - lo > width ? hi - width : lo;
  }
  __syncthreads();
  Place p;
  p.key = hi;
  p.n = n;
  p.eq = count;
  p.index = -1;
  p.m = m;
  p.w = (double)w.mass(value_of(hi), (float)b) * unit;
  p.at = which_of(q, n, m, p.w, count);
  return p;
}

// the index of the at-th token (by index) of the logit `key`
template <class E>
__device__ int index_of(const typename E::t* row, int V, const Place& p, Shared& s) {
  if (p.index >= 0) return p.index;
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6;
  __syncthreads();
  if (t < 64) s.slab[t] = 0;
  if (t == 0) s.token = -1;
  __syncthreads();
  // 64 slabs of whole vectors
  const int slab = ((V + 63) / 64 + 7) / 8 * 8;
  each<E>(row, V, [&](float z, int i) {
    if (key_of(z) == p.key) {
      if (p.eq == 1) s.token = i;
      else atomicAdd(&s.slab[i / slab], 1u);
    }
  });
  __syncthreads();
  if (p.eq == 1) return s.token;
  uint32_t before = 0;
  int c = 0;
  for (; c < 63 && before + s.slab[c] <= p.at; ++c) before += s.slab[c];
  // in order inside the slab, 1024 tokens at a time
  const int lo = c * slab, hi = min(V, lo + slab);
  for (int i0 = lo; i0 < hi; i0 += kThreads) {
    const int i = i0 + t;
    const bool eq = i < hi && key_of(E::one(row + i) + 0.f) == p.key;
    const unsigned long long bal = __ballot(eq);
    __syncthreads();
    if (lane == 0) s.wave_in[wid] = __popcll(bal);
    __syncthreads();
    uint32_t mine = before + __popcll(bal & ((1ull << lane) - 1ull));
    for (int v = 0; v < kWaves; ++v) {
      mine += v < wid ? s.wave_in[v] : 0;
      before += s.wave_in[v];
    }
    if (eq && mine == p.at) s.token = i;
  }
  __syncthreads();
  return s.token;
}

// a row of any type and length, read from memory in each pass
template <class E>
__device__ __forceinline__ void sample_row(const SampleCall& a, int n, Shared& s) {
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6, V = a.V;
  const typename E::t* row = static_cast<const typename E::t*>(a.logits) + n * a.stride;
  typename E::t* out = a.filtered ? static_cast<typename E::t*>(a.filtered) + n * a.filtered_stride : nullptr;
  const float scale = a.scales ? a.scales[n] : a.scale;
  const int top_k = a.top_ks ? a.top_ks[n] : a.top_k;
  const float top_p = a.top_ps ? a.top_ps[n] : a.top_p, min_p = a.min_ps ? a.min_ps[n] : a.min_p;

  // the maximum; NaN, and +inf, leave no distribution
  float top = -INFINITY;
  each_eight<E>(row, V, [&](auto& z, int) __attribute__((always_inline)) { top = largest(top, z); });
  bool bad = top != top;
  top += 0.f;   // (of zeros the positive one)
  // Of a short list (top_k): a sixteenth of it, the j-th largest of the lanes' own best, bit by bit: of the lanes that
  // agree with it so far, those with a 1 come first. The worst of the waves' is a bound for the whole list.
  uint32_t bound = 0;
  const bool few = top_k > 0 && top_k <= kThreads;
  if (few) {
    const uint32_t own = key_of(top);
    int j = (top_k + kWaves - 1) / kWaves;
    unsigned long long left = ~0ull;
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned long long ones = left & __ballot(own >> bit & 1);
      const int c = __popcll(ones);
      if (j <= c) {
        left = ones;
        bound |= 1u << bit;
      } else {
        left &= ~ones;
        j -= c;
      }
    }
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));   // (NaN is in `bad`)
  const bool any_bad = __any(bad);
  if (lane == 0) {
    s.wave_top[wid] = top;
    s.wave_bad[wid] = any_bad;
    s.wave_in[wid] = bound;
  }
  for (uint32_t i = t; i < sizeof(s.copies) / 16; i += kThreads) reinterpret_cast<u32x4*>(s.copies)[i] = u32x4{0u, 0u, 0u, 0u};
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    top = fmaxf(top, s.wave_top[w]);
    bad |= s.wave_bad[w] != 0;
  }
  const float sc = scale == 0.f ? 1.f : scale;
  if (bad || !(fabsf(top) < INFINITY) || !(sc > 0.f && sc <= kSampleMaxScale)) {
    if (t == 0) {
      a.token[n] = -1;
      if (a.prob) a.prob[n] = NAN;
      if (a.kept) a.kept[n] = 0;
    }
    if (out)
      for (int i = t; i < V; i += kThreads) out[i] = E::to(-INFINITY);
    return;
  }
  const Weigh w(top, sc);
  const uint32_t key_top = key_of(top);
  const bool least = min_p > 0.f;
  const double limit = least ? -log(fmin((double)min_p, 1.0)) : 0.0;   // nats below the maximum
  // What cannot be kept is not counted: what min_p alone leaves out (`limit` and a little more), and of a short list what
  // is below the worst of the waves' bounds.
  uint32_t from = key_of(-3.402823466e38f);
  if (least && top_k <= 0 && !(top_p < 1.f)) from = max(from, key_of((float)((double)top - (limit + 0.03) / w.scale)));
  if (few) {
    bound = ~0u;
    for (int v = 0; v < kWaves; ++v) bound = min(bound, s.wave_in[v]);
    from = max(from, bound);
  }
  const bool list = from > key_of(-3.402823466e38f);   // then they are few, and listed at once
  if (t == 0) {
    s.listed = 0;
    s.from = from;
  }
  __syncthreads();
  uint32_t inside = 0, infs = 0;
  Counts& counts = s.copies[lane & 3];
  const float above = value_of(from);
  auto add = [&](float z) __attribute__((always_inline)) {
    const float b = w.bin_of(z);
    atomicAdd(&counts.n[(int)b], 1u);   // (-inf in the last bin, subtracted below)
    atomicAdd(&counts.mass[(int)b], w.mass(z, b));   // (of the last bin anything: it is worth nothing)
    if (least) inside += w.below(z) <= limit;
  };
  each_eight<E>(row, V, [&](auto& z, int i) __attribute__((always_inline)) {
    constexpr int N = sizeof(z) / sizeof(float);
    if (smallest(z) == -INFINITY) {
#pragma unroll
      for (int e = 0; e < N; ++e) infs += z[e] == -INFINITY;
    }
    if (!list) {
#pragma unroll
      for (int e = 0; e < N; ++e) add(z[e]);
    } else if (largest(z[0], z) >= above) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float y = z[e] + 0.f;
        if (y >= above) {
          const uint32_t at = atomicAdd(&s.listed, 1u);
          if (at < kListed) {
            s.list_key[at] = key_of(y);
            s.list_index[at] = i + e;
          }
        }
      }
    }
  });
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) infs += __shfl_xor(infs, k);
  if (lane == 0) s.wave_n[wid] = infs;
  __syncthreads();
  infs = 0;
  for (int v = 0; v < kWaves; ++v) infs += s.wave_n[v];
  uint32_t kept = V - infs;
  if (list && short_enough(s.listed, kept, top_k)) {
    if (out)
      for (int i = t; i < V; i += kThreads) out[i] = E::to(-INFINITY);
    const uint32_t key = s.list_key[t];   // (of the listed only)
    const int index = s.list_index[t];
    uint32_t rank;
    const uint32_t seen = s.listed;
    const uint32_t n_kept = draw_short(s.few, a, n, w, Filters{top_k, top_p, a.r[n], least, limit}, seen,
                                       top_k > 0 ? kept : seen, ~key, index, value_of(key), rank);
    if (out && t < (int)seen && rank < n_kept) out[index] = row[index];
    return;
  }
  if (list && s.listed <= kListed)
    for (uint32_t i = t; i < s.listed; i += kThreads) add(value_of(s.list_key[i]));
  else if (list)
    each<E>(row, V, [&](float z, int) {
      if (z >= above) add(z);
    });
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) inside += __shfl_xor(inside, k);
  if (lane == 0) s.wave_in[wid] = inside;
  __syncthreads();
  inside = 0;
  for (int v = 0; v < kWaves; ++v) inside += s.wave_in[v];
  if (t == 0) {
    s.list_lo = list && s.listed <= kListed ? from : 1;
    s.list_hi = list && s.listed <= kListed ? key_top : 0;
  }
  for (int i = t; i < kBins; i += kThreads) {
    uint32_t c = 0;
    unsigned long long m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c += s.copies[k].n[i];
      m += s.copies[k].mass[i];
    }
    s.copies[0].n[i] = i == kFar && !list ? c - infs : c;   // those of `all`
    s.copies[0].mass[i] = m;
  }
  __syncthreads();
  scan<true>(s.all, 0.0, s);

  double mass = s.all.m_upto[kBins - 1];
  Place cut{};
  bool is_cut = false;
  // top_k, top_p, min_p, the draw
  Place p{};
  for (int step = 0; step < 4; ++step) {
    Bound q{};
    if (step == 0) {
      if (top_k <= 0 || (uint32_t)top_k >= kept) continue;
      q = Bound{true, false, (uint32_t)top_k - 1, 0.0};
    } else if (step == 1) {
      if (!(top_p < 1.f)) continue;
      q = Bound{false, true, 0, fmax((double)top_p, 0.0) * mass};
    } else if (step == 2) {
      if (!least || inside >= kept) continue;
      q = Bound{true, false, inside - 1, 0.0};
    } else {
      q = Bound{false, false, 0, fmin(fmax((double)a.r[n], 0.0), 1.0) * mass};
    }
    p = find<E>(row, V, w, key_top, q, s);
    if (step < 3 && p.rank() + 1 < kept) {
      cut = p;
      is_cut = true;
      kept = p.rank() + 1;
      mass = p.upto();
    }
  }
  if (is_cut && p.rank() > cut.rank()) p = cut;   // by rounding alone
  const int token = index_of<E>(row, V, p, s);
  if (t == 0) {
    a.token[n] = token;
    if (a.prob) a.prob[n] = (float)(p.w / mass);
    if (a.kept) a.kept[n] = (int)kept;
  }
  if (!out) return;
  uint32_t key = 0;
  int last = V;   // of the tokens of that key
  if (is_cut) {
    key = cut.key;
    if (cut.at + 1 < cut.eq) last = index_of<E>(row, V, cut, s);
  }
  each<E>(row, V, [&](float z, int i) {
    const uint32_t k = key_of(z);
    out[i] = k > key || (k == key && i <= last) ? row[i] : E::to(-INFINITY);
  });
}

// the same where it is rare
template <class E>
__device__ __noinline__ void sample_row_apart(const SampleCall a, int n, Shared& s) {
  sample_row<E>(a, n, s);
}
template <class E>
__global__ __launch_bounds__(kThreads) void k_sample(SampleCall a) {
  __shared__ Shared s;
  sample_row<E>(a, blockIdx.x, s);
}

// ------------------------------------------------- 16-bit logits, held in registers --
//
// A row of up to 163840 logits of 16 bits fits a workgroup's registers, and a
// table with a 16-bit count for each of the 65536 values fits its LDS. (256
// rows of 126464 with top_p take 32 us here, 32 of 152064 with the filtered
// logits written 36 to 42, 256 of 32000 16; the other way 57, 92 and 39.) So the
// row is read once and counted by value, one LDS addition a token; masses are
// then counts times the exponential of a value, and no token needs one of its
// own. A thread sums the 64 values of its block of the table (equally spaced:
// they share an exponent, so their exponentials are a geometric series, one
// multiply-add each); bounds are found by the first wave alone, in the blocks'
// running sums and then in a block, a value a lane.
//
// Values are slots, falling as they rise: 0 .. 0x7fff the positive ones from
// the largest down, 0x8000 .. the negative ones. What is 64 nats and more below
// the maximum has no mass (e^-64 of it) and is not counted.

template <class E>
struct Slots;
template <>
struct Slots<Bf16> {
  static constexpr uint32_t low = 0xff80;   // of -inf
};
template <>
struct Slots<F16> {
  static constexpr uint32_t low = 0xfc00;
};
constexpr uint32_t kZero = 0x7fff, kMinusZero = 0x8000;

template <class E>
__device__ __forceinline__ float slot_value(uint32_t s) {
  const uint16_t b = (uint16_t)(s & 0x8000 ? s : s ^ 0x7fff);
  return E::one(&b);
}
template <class E>
__device__ __forceinline__ uint32_t slot_of(float z) {
  const uint32_t b = E::to(z);
  return b & 0x8000 ? b : b ^ 0x7fff;
}
// both halves
__device__ __forceinline__ uint32_t slots_of(uint32_t w) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, w) >> (short)15);
  return (sign & w) | (~sign & (w ^ 0x7fff7fffu));
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct KeyPlace {   // as Place, with a slot in place of the key
  uint32_t slot, n, eq, at;
  double m, w;
  __device__ __forceinline__ uint32_t rank() const { return n + at; }
  __device__ __forceinline__ double upto() const { return m + (double)(at + 1) * w; }
};

constexpr int kCounted = 2 * kThreads;   // as many as fit beside the table

struct Keys {
  uint32_t count[32768];   // of slot s in word s % 32768: the positive values in the low halves, the negative in the high ones
  uint32_t n_upto[kThreads];
  double m_upto[kThreads];
  uint32_t wave_n[kWaves];
  double wave_m[kWaves];
  uint32_t wave_lo[kWaves], wave_hi[kWaves];
  KeyPlace cut, pick;
  int is_cut, give_up, token;
  uint32_t kept;
  double mass;
  uint32_t slab[64];
  uint32_t listed, list_slot[kCounted];   // the counted tokens, where they are few
  int list_index[kCounted];
};

__device__ __forceinline__ uint32_t count_of(const Keys& s, uint32_t slot) {
  const uint32_t w = s.count[slot & 0x7fff];
  return slot & 0x8000 ? w >> 16 : w & 0xffff;
}

// By the first wave: the token at which a bound is passed.
template <class E>
__device__ __forceinline__ KeyPlace find_key(const Keys& s, const Weigh& w, const Bound& q) {
  const int lane = threadIdx.x & 63;
  // 64 blocks of the 16 times 64, the block, the value
  const int g = lane & 15;
  const int group = first_of(q, s.n_upto[g * 64 + 63], s.m_upto[g * 64 + 63], g ? s.n_upto[g * 64 - 1] : 0, lane < 16);
  const int b0 = group * 64 + lane;
  const int b = group * 64 + first_of(q, s.n_upto[b0], s.m_upto[b0], b0 ? s.n_upto[b0 - 1] : 0, true);
  const uint32_t n0 = b ? s.n_upto[b - 1] : 0;
  const double m0 = b ? s.m_upto[b - 1] : 0.0;
  const uint32_t slot = b * 64 + lane, c = count_of(s, slot);
  const double e = c ? exp(-w.below(slot_value<E>(slot))) : 0.0;
  const uint32_t n = n0 + wave_scan(c);
  const double m = m0 + wave_scan((double)c * e);
  const int at = first_of(q, n, m, n - c, true);
  KeyPlace p;
  p.slot = b * 64 + at;
  p.eq = __builtin_amdgcn_readlane(c, at);
  p.n = __builtin_amdgcn_readlane(n, at) - p.eq;
  p.m = at ? lane_of(m, at - 1) : m0;
  p.w = lane_of(e, at);
  p.at = which_of(q, p.n, p.m, p.w, p.eq);
  return p;
}

// NV: vectors of 8 tokens a thread, without the row's last 8192 (at most)
template <class E, int NV>
__global__ __launch_bounds__(kThreads) void k_sample_keys(SampleCall a) {
  constexpr size_t kBytes = sizeof(Keys) > sizeof(Shared) ? sizeof(Keys) : sizeof(Shared);
  __shared__ __attribute__((aligned(16))) unsigned char lds[kBytes];
  Keys& s = *reinterpret_cast<Keys*>(lds);
  constexpr uint32_t kLow = Slots<E>::low;
  const int n = blockIdx.x, t = threadIdx.x, lane = t & 63, wid = t >> 6, V = a.V;
  const typename E::t* row = static_cast<const typename E::t*>(a.logits) + n * a.stride;
  const float scale = a.scales ? a.scales[n] : a.scale;
  const int top_k = a.top_ks ? a.top_ks[n] : a.top_k;
  const float top_p = a.top_ps ? a.top_ps[n] : a.top_p, min_p = a.min_ps ? a.min_ps[n] : a.min_p;

  // vector j holds tokens 8 (t + 1024 j) .., the tail what is left, `tails` of them; its other places a token again that
  // the thread holds already, if it holds any
  uint32_t v[NV][4], tail[4];
  const int steps = (V - 1) / (8 * kThreads), tail_at = 8 * (t + steps * kThreads), tails = min(max(V - tail_at, 0), 8);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (j < steps) x = reinterpret_cast<const Any16*>(row + 8 * (t + j * kThreads))->v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[j][e] = x[e];
  }
  if (tails == 8) {
    const u32x4 x = reinterpret_cast<const Any16*>(row + tail_at)->v;
#pragma unroll
    for (int e = 0; e < 4; ++e) tail[e] = x[e];
  } else {
    const uint32_t some = tails > 0 ? row[tail_at] : steps > 0 ? v[0][0] & 0xffff : row[0];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      tail[e] = (2 * e < tails ? row[tail_at + 2 * e] : some) | (2 * e + 1 < tails ? row[tail_at + 2 * e + 1] : some) << 16;
  }
  for (int i = t; i < 8192; i += kThreads) reinterpret_cast<u32x4*>(s.count)[i] = u32x4{0u, 0u, 0u, 0u};
  if (t == 0) s.give_up = s.listed = 0;
  u16x2 lo = {0xffff, 0xffff}, hi = {0, 0};
  auto take = [&](uint32_t& x) __attribute__((always_inline)) {
    x = slots_of(x);
    asm("" : "+v"(x));   // kept in place of what it came from
    lo = __builtin_elementwise_min(lo, __builtin_bit_cast(u16x2, x));
    hi = __builtin_elementwise_max(hi, __builtin_bit_cast(u16x2, x));
  };
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j < steps) {
#pragma unroll
      for (int e = 0; e < 4; ++e) take(v[j][e]);
    }
#pragma unroll
  for (int e = 0; e < 4; ++e) take(tail[e]);
  const uint32_t mine = min((uint32_t)lo.x, (uint32_t)lo.y);
  uint32_t first = mine, last = max((uint32_t)hi.x, (uint32_t)hi.y);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    first = min(first, (uint32_t)__shfl_xor((int)first, k));
    last = max(last, (uint32_t)__shfl_xor((int)last, k));
  }
  // Of a short list (top_k): a sixteenth of it, the j-th smallest of the lanes' slots, bit by bit: of the lanes that agree
  // with it so far, those with a 0 come first. The worst of the waves' is a bound for the whole list.
  // (Not of longer ones: of 126464 tokens top_k of 200 takes 22.6 us so and 300 24.2, counting all of them 23.5. The
  // filtered row is quicker written from a list: 32 rows of 152064 with lists of up to 472 take 36 us so, 44 counting all.)
  uint32_t bound = 0;
  const bool few = top_k > 0 && top_k <= (a.filtered ? 512 : 256);
  if (few) {
    const uint32_t own = tails == 0 && steps == 0 ? kLow : mine;   // a lane without a token of its own
    int j = (top_k + kWaves - 1) / kWaves;
    unsigned long long left = ~0ull;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
      const unsigned long long zeros = left & ~__ballot(own >> bit & 1);
      const int c = __popcll(zeros);
      if (j <= c) {
        left = zeros;
      } else {
        left &= ~zeros;
        j -= c;
        bound |= 1u << bit;
      }
    }
  }
  if (lane == 0) {
    s.wave_lo[wid] = first;
    s.wave_hi[wid] = last;
    s.wave_n[wid] = bound;
  }
  __syncthreads();
  bound = 0;
  for (int k = 0; k < kWaves; ++k) {
    first = min(first, s.wave_lo[k]);
    last = max(last, s.wave_hi[k]);
    bound = max(bound, s.wave_n[k]);
  }
  first = __builtin_amdgcn_readfirstlane(first == kMinusZero ? kZero : first);
  last = __builtin_amdgcn_readfirstlane(last);
  const float top = slot_value<E>(first), sc = scale == 0.f ? 1.f : scale;
  // NaN (on either side) or +inf in the row, nothing but -inf, or no temperature
  if (last > kLow || first >= kLow || !(fabsf(top) < INFINITY) || !(sc > 0.f && sc <= kSampleMaxScale)) {
    __syncthreads();
    sample_row_apart<E>(a, n, *reinterpret_cast<Shared*>(lds));
    return;
  }
  const Weigh w(top, sc);
  const bool least = min_p > 0.f;
  const double limit = least ? -log(fmin((double)min_p, 1.0)) : 0.0;   // nats below the maximum
  // Slots beyond `end` are not counted: 64 nats below; of min_p alone, what it leaves out (`limit` and a little more); of
  // a short list, what no token of it can be.
  const bool min_alone = least && top_k <= 0 && !(top_p < 1.f);
  const double reach = min_alone ? fmin(limit + 0.03, 64.0) : 64.0;
  uint32_t end = min(slot_of<E>((float)((double)top - reach / (double)sc)), kLow - 1);
  if (few) end = min(end, bound);
  end = __builtin_amdgcn_readfirstlane(end == kZero ? kMinusZero : end);   // -0 is equal
  uint32_t infs = 0, seen = V;   // -inf, and what was counted
  auto count = [&](uint32_t x) __attribute__((always_inline)) {
    atomicAdd(&s.count[x & 0x7fff], 1u + (x >> 15) * 0xffffu);
  };
  typename E::t* out = a.filtered ? static_cast<typename E::t*>(a.filtered) + n * a.filtered_stride : nullptr;
  bool listed = false;
  // (comparisons of the number of vectors are cheap to repeat, but kept from one loop to the next they fill the registers)
  auto again = [&] {
    int x = steps;
    asm("" : "+s"(x));
    return x;
  };
  if (last <= end) {   // everything
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j < steps) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          count(v[j][e] & 0xffff);
          count(v[j][e] >> 16);
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // one vector at a time: the row takes most of the registers
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (2 * e < tails) count(tail[e] & 0xffff);
      if (2 * e + 1 < tails) count(tail[e] >> 16);
    }
  } else {
    uint32_t in = 0, inf = 0;
    auto low_half = [](uint32_t x) { return x & 0xffff; };
    auto least_of = [](const uint32_t (&x)[4]) {
      u16x2 m = {0xffff, 0xffff};
#pragma unroll
      for (int e = 0; e < 4; ++e) m = __builtin_elementwise_min(m, __builtin_bit_cast(u16x2, x[e]));
      return min((uint32_t)m.x, (uint32_t)m.y);
    };
    auto infs_of = [&](const uint32_t (&x)[4], int tokens) __attribute__((always_inline)) {
      if (last != kLow) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) inf += (e & 1 ? x[e >> 1] >> 16 : low_half(x[e >> 1])) == kLow && e < tokens;
    };
    if (few || min_alone) {
      auto take = [&](uint32_t y, int i) __attribute__((always_inline)) {
        const uint32_t at = atomicAdd(&s.listed, 1u);
        if (at < kCounted) {
          s.list_slot[at] = y;
          s.list_index[at] = i;
        }
      };
      auto vector = [&](const uint32_t (&x)[4], int i0, int tokens) __attribute__((always_inline)) {
        if (least_of(x) <= end) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y0 = low_half(x[e]), y1 = x[e] >> 16;
            if (min(y0, y1) <= end) {
              if (y0 <= end && 2 * e < tokens) take(y0, i0 + 2 * e);
              if (y1 <= end && 2 * e + 1 < tokens) take(y1, i0 + 2 * e + 1);
            }
          }
        }
        infs_of(x, tokens);
      };
      const int held = again();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j < held) vector(v[j], 8 * (t + j * kThreads), 8);
        __builtin_amdgcn_sched_barrier(0);
      }
      vector(tail, tail_at, tails);
      __syncthreads();
      seen = __builtin_amdgcn_readfirstlane(s.listed);
      listed = seen <= kCounted;
    }
    if (!listed) {
      auto vector = [&](const uint32_t (&x)[4], int tokens) __attribute__((always_inline)) {
        if (least_of(x) <= end) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t y = e & 1 ? x[e >> 1] >> 16 : low_half(x[e >> 1]);
            if (y <= end && e < tokens) {
              count(y);
              ++in;
            }
          }
        }
        infs_of(x, tokens);
      };
      inf = 0;
      const int held = again();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j < held) vector(v[j], 8);
        __builtin_amdgcn_sched_barrier(0);
      }
      vector(tail, tails);
    }
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) {
      inf += __shfl_xor(inf, k);
      in += __shfl_xor(in, k);
    }
    __syncthreads();
    if (lane == 0) {
      s.wave_n[wid] = inf;
      s.wave_hi[wid] = in;
    }
    __syncthreads();
    if (!listed) seen = 0;
    for (int k = 0; k < kWaves; ++k) {
      infs += s.wave_n[k];
      seen += s.wave_hi[k];
    }
    seen = __builtin_amdgcn_readfirstlane(seen);
    // then nearly all that is filtered is -inf: written now, beside what follows, and the kept ones over it
    if (listed && out) {
      const uint32_t gone = (uint32_t)E::to(-INFINITY) * 0x10001u;
#pragma unroll 1
      for (int j = 0; j < steps; ++j)
        reinterpret_cast<Any16*>(out + 8 * (t + j * kThreads))->v = u32x4{gone, gone, gone, gone};
#pragma unroll 1
      for (int e = 0; e < tails; ++e) out[tail_at + e] = (typename E::t)gone;
    }
  }
  __syncthreads();
  const uint32_t finite = V - infs;
  const bool low = least && limit > 63.0;   // what min_p keeps may not have been counted
  if (listed && !low && short_enough(seen, finite, top_k)) {
    const uint32_t x = s.list_slot[t];   // (of the listed only)
    const int index = s.list_index[t];
    uint32_t rank;
    const uint32_t kept = draw_short(*reinterpret_cast<Short*>(s.count), a, n, w, Filters{top_k, top_p, a.r[n], least, limit},
                                     seen, top_k > 0 ? finite : seen, x == kMinusZero ? kZero : x, index, slot_value<E>(x), rank);
    if (out && t < (int)seen && rank < kept) out[index] = (typename E::t)(x & 0x8000 ? x : x ^ 0x7fff);
    return;
  }
  if (listed) {
    for (uint32_t i = t; i < seen; i += kThreads) count(s.list_slot[i]);
    __syncthreads();
  }
  if (t == 0) {   // the two zeros are equal
    const uint32_t minus = count_of(s, kMinusZero);
    if (minus) {
      if (count_of(s, kZero) + minus > 0xffff) s.give_up = 1;
      s.count[kZero] += minus;
      s.count[0] -= minus << 16;
    }
  }
  __syncthreads();
  // Four lanes a block of 64 values, 16 values each: equally spaced by u, so the masses are e_0 rho^i.
  for (int r = 0; r < 4; ++r) {
    const int at = (r * kThreads + t) * 16, half = at & 0x8000 ? 16 : 0;
    const u32x4* p = reinterpret_cast<const u32x4*>(&s.count[at & 0x7fff]);
    uint32_t any = 0, bn = 0;
    const uint32_t from = (uint32_t)(r * kThreads + wid * 64) * 16;   // of the wave's first lane
    if (from <= end && from + 1024 > first) {
      // lanes are 64 bytes apart: beginning at another quarter each, they meet all banks
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 c = p[(j + (t >> 2)) & 3];
        any |= c[0] | c[1] | c[2] | c[3];
      }
    }
    double bm = 0.0;
    if (any >> half & 0xffff) {
      const float z0 = slot_value<E>(at), u = z0 - slot_value<E>(at + 1);
      const double per = -(double)u * w.scale, d0 = -w.below(z0);
      if (d0 > 600.0) s.give_up = 1;   // so steep that the values above the maximum in its block overflow
      const double e0 = exp(d0), rho = exp(per), rho2 = rho * rho;
      double even = 0.0, odd = 0.0;
      u32x4 c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = p[j];
#pragma unroll
      for (int i = 14; i >= 0; i -= 2) {
        const uint32_t x = c[i >> 2][i & 3] >> half & 0xffff, y = c[i >> 2][(i & 3) + 1] >> half & 0xffff;
        bn += x + y;
        even = fma(even, rho2, (double)x);
        odd = fma(odd, rho2, (double)y);
      }
      bm = fma(odd, rho, even) * e0;
    }
    bn += __shfl_xor(bn, 1);
    bm += __shfl_xor(bm, 1);
    bn += __shfl_xor(bn, 2);
    bm += __shfl_xor(bm, 2);
    if ((t & 3) == 0) {
      s.n_upto[at >> 6] = bn;
      s.m_upto[at >> 6] = bm;
    }
  }
  __syncthreads();
  const uint32_t un = wave_scan(s.n_upto[t]);
  const double um = wave_scan(s.m_upto[t]);
  if (lane == 63) {
    s.wave_lo[wid] = un;
    s.wave_m[wid] = um;
  }
  __syncthreads();
  uint32_t counted = 0, base_n = 0;
  double base_m = 0.0;
  for (int k = 0; k < kWaves; ++k) {
    base_n += k < wid ? s.wave_lo[k] : 0;
    base_m += k < wid ? s.wave_m[k] : 0.0;
    counted += s.wave_lo[k];
  }
  s.n_upto[t] = base_n + un;
  s.m_upto[t] = base_m + um;
  __syncthreads();
  // A count that ran over its 16 bits shows in their sum. Those, and ranks among what is not counted, are rare and left
  // to the other way.
  const bool far = top_k > 0 && (uint32_t)top_k > counted && (uint32_t)top_k < finite;
  if (seen != counted || s.give_up || far || low) {
    __syncthreads();
    sample_row_apart<E>(a, n, *reinterpret_cast<Shared*>(lds));
    return;
  }
  if (wid == 0) {
    uint32_t kept = finite;
    double mass = s.m_upto[kThreads - 1];
    KeyPlace cut{};
    bool is_cut = false;
    if (top_k > 0 && (uint32_t)top_k < kept) {
      cut = find_key<E>(s, w, Bound{true, false, (uint32_t)top_k - 1, 0.0});
      is_cut = true;
      kept = top_k;
      mass = cut.upto();
    }
    if (top_p < 1.f) {
      const KeyPlace p = find_key<E>(s, w, Bound{false, true, 0, fmax((double)top_p, 0.0) * mass});
      if (p.rank() + 1 < kept) {
        cut = p;
        is_cut = true;
        kept = p.rank() + 1;
        mass = p.upto();
      }
    }
    if (least) {
      // the blocks whose first value min_p leaves, then the values of the last of them
      auto leaves = [&](uint32_t slot) {
        return w.below(slot_value<E>(min(max(slot, first), kLow - 1))) <= limit;
      };
      const int group = __popcll(__ballot(lane < 16 && leaves(lane * 4096))) - 1;
      const int b = group * 64 + __popcll(__ballot(leaves(group * 4096 + lane * 64))) - 1;
      const uint32_t slot = b * 64 + lane, c = count_of(s, slot);
      uint32_t in = c && leaves(slot) ? c : 0;
#pragma unroll
      for (int k = 32; k >= 1; k >>= 1) in += __shfl_xor(in, k);
      in += b ? s.n_upto[b - 1] : 0;
      if (in < kept) {
        cut = find_key<E>(s, w, Bound{true, false, in - 1, 0.0});
        is_cut = true;
        kept = in;
        mass = cut.upto();
      }
    }
    KeyPlace p = find_key<E>(s, w, Bound{false, false, 0, fmin(fmax((double)a.r[n], 0.0), 1.0) * mass});
    if (is_cut && p.rank() > cut.rank()) p = cut;   // by rounding alone
    if (lane == 0) {
      s.pick = p;
      s.cut = cut;
      s.is_cut = is_cut;
      s.kept = kept;
      if (a.prob) a.prob[n] = (float)(p.w / mass);
      if (a.kept) a.kept[n] = (int)kept;
    }
  }
  // the index of the at-th token of a slot: in order of the vectors, then of the threads, then inside the vector
  auto index_of = [&](const KeyPlace& p) __attribute__((always_inline)) {
    __syncthreads();
    const uint32_t slot = __builtin_amdgcn_readfirstlane(p.slot), eq = __builtin_amdgcn_readfirstlane(p.eq),
                   at = __builtin_amdgcn_readfirstlane(p.at);
    const bool zero = slot == kZero;
    if (t == 0) {
      s.token = -1;
      s.wave_n[0] = 0;
    }
    if (t <= NV) s.slab[t] = 0;
    __syncthreads();
    auto same = [&](uint32_t x) __attribute__((always_inline)) { return x == slot || (zero && x == kMinusZero); };
    if (listed && eq <= 64) {   // among the listed: s.slab[0 ..] takes the indexes of the equal ones
      for (uint32_t i = t; i < seen; i += kThreads)
        if (same(s.list_slot[i])) {
          if (eq == 1) s.token = s.list_index[i];
          else s.slab[atomicAdd(&s.wave_n[0], 1u)] = s.list_index[i];
        }
      if (eq > 1) {
        __syncthreads();
        if (t < (int)eq) {   // each sees how many lie before it
          uint32_t before = 0;
          for (uint32_t k = 0; k < eq; ++k) before += s.slab[k] < s.slab[t];
          if (before == at) s.token = s.slab[t];
        }
      }
      __syncthreads();
      return s.token;
    }
    auto matches = [&](const uint32_t (&x)[4], int tokens) __attribute__((always_inline)) {   // a bit a token
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m |= (uint32_t)(same(e & 1 ? x[e >> 1] >> 16 : x[e >> 1] & 0xffff) && e < tokens) << e;
      return m;
    };
    // a few equal ones are gathered; more are counted in slabs, a vector each, and sought in one of them
    const bool gather = !listed && eq <= 256;
    auto vector = [&](const uint32_t (&x)[4], int j, int tokens) __attribute__((always_inline)) {
      // a half that is equal leaves 0 in place of 1
      auto differ = [&](uint32_t key) __attribute__((always_inline)) {
        uint32_t r = 0x10001u;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          r &= __builtin_bit_cast(uint32_t,
                                  __builtin_elementwise_min(__builtin_bit_cast(u16x2, x[e] ^ key * 0x10001u), u16x2{1, 1}));
        return r;
      };
      uint32_t d = differ(slot);
      if (zero) d &= differ(kMinusZero);
      if (d != 0x10001u) {
        uint32_t m = matches(x, tokens);
        const int i0 = 8 * (t + j * kThreads);
        if (eq == 1) {
          if (m) s.token = i0 + __builtin_ctz(m);
        } else if (gather) {
          for (; m; m &= m - 1) s.list_index[atomicAdd(&s.wave_n[0], 1u)] = i0 + __builtin_ctz(m);
        } else if (m) {
          atomicAdd(&s.slab[j < steps ? j : NV], __popc(m));
        }
      }
    };
    const int held = again();
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j < held) vector(v[j], j, 8);
    vector(tail, steps, tails);
    __syncthreads();
    if (eq > 1 && gather) {   // each sees how many lie before it
      if (t < (int)eq) {
        const int index = s.list_index[t];
        uint32_t before = 0;
#pragma unroll 4
        for (uint32_t k = 0; k < eq; ++k) before += s.list_index[k] < index;
        if (before == at) s.token = index;
      }
      __syncthreads();
    } else if (eq > 1) {
      uint32_t before = 0;
      int slab = 0;   // NV: the tail
      for (; slab < NV && before + s.slab[slab] <= at; ++slab) before += s.slab[slab];
      uint32_t m = slab == NV ? matches(tail, tails) : 0;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (j == slab) m = matches(v[j], 8);
      const uint32_t c = __popc(m), upto = wave_scan(c);
      if (lane == 63) s.wave_n[wid] = upto;
      __syncthreads();
      for (int k = 0; k < wid; ++k) before += s.wave_n[k];
      before += upto - c;
      if (at >= before && at < before + c) {
        for (uint32_t i = before; i < at; ++i) m &= m - 1;
        s.token = 8 * (t + (slab == NV ? steps : slab) * kThreads) + __builtin_ctz(m);
      }
      __syncthreads();
    }
    return s.token;
  };
  __syncthreads();
  const int token = index_of(s.pick);
  if (t == 0) a.token[n] = token;
  if (!out) return;
  // what comes before the cut's slot stays, and of its tokens those up to the last kept one
  const bool is_cut = s.is_cut;
  uint32_t slot = __builtin_amdgcn_readfirstlane(is_cut ? s.cut.slot : kLow);
  int until = V;
  if (is_cut && s.cut.at + 1 < s.cut.eq) until = __builtin_amdgcn_readfirstlane(index_of(s.cut));
  const uint32_t after = slot == kZero ? kMinusZero : slot;
  if (listed && s.kept <= seen) {   // (else some are kept that were not counted, of no mass)
    for (uint32_t k = t; k < seen; k += kThreads) {
      const uint32_t x = s.list_slot[k], i = s.list_index[k];
      if (x <= after && !(x >= slot && (int)i > until)) out[i] = (typename E::t)(x & 0x8000 ? x : x ^ 0x7fff);
    }
    return;
  }
  const uint32_t gone = (uint32_t)E::to(-INFINITY) * 0x10001u;
  auto left = [&](const uint32_t (&x)[4], int i0) __attribute__((always_inline)) {
    u32x4 o = {gone, gone, gone, gone};
    u16x2 m = {0xffff, 0xffff};
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __builtin_elementwise_min(m, __builtin_bit_cast(u16x2, x[e]));
    const uint32_t bound = i0 > until ? slot - 1 : after;
    if (min((uint32_t)m.x, (uint32_t)m.y) > bound) return o;   // most, in most rows
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // halves above the bound go: 0xffff there
      const u16x2 y = __builtin_bit_cast(u16x2, x[e]);
      const u16x2 over = y ^ __builtin_elementwise_min(y, u16x2{(unsigned short)bound, (unsigned short)bound});
      uint32_t drop = __builtin_bit_cast(uint32_t, u16x2{0, 0} - __builtin_elementwise_min(over, u16x2{1, 1}));
      if ((uint32_t)(until - i0) < 8u) {   // the last kept one of the cut's own is in here
        const uint32_t x0 = x[e] & 0xffff, x1 = x[e] >> 16;
        drop |= x0 >= slot && i0 + 2 * e > until ? 0xffffu : 0;
        drop |= x1 >= slot && i0 + 2 * e + 1 > until ? 0xffff0000u : 0;
      }
      o[e] = (drop & gone) | (~drop & slots_of(x[e]));   // (its own inverse)
    }
    return o;
  };
  const int held = again();
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j < held) reinterpret_cast<Any16*>(out + 8 * (t + j * kThreads))->v = left(v[j], 8 * (t + j * kThreads));
  const u32x4 o = left(tail, tail_at);
  if (tails == 8) {
    reinterpret_cast<Any16*>(out + tail_at)->v = o;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < tails) out[tail_at + e] = (typename E::t)(o[e >> 1] >> (16 * (e & 1)));
  }
}

// The fewest vectors that hold the row: places for vectors that it does not have are skipped, but cost registers and code.
// 256 rows of bf16 with top_p: 8000 tokens 13 us, in the form for the longest rows 18; 32000 16 and 21, 65000 22 and 27,
// 126464 32 and 37.
template <class E>
void sample_keys(const SampleCall& a, hipStream_t s) {
  constexpr int kStep = 8 * kThreads;
  if (a.V <= 5 * kStep)
    k_sample_keys<E, 4><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 10 * kStep)
    k_sample_keys<E, 9><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 16 * kStep)
    k_sample_keys<E, 15><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 20 * kStep)
    k_sample_keys<E, 19><<<a.N, kThreads, 0, s>>>(a);
  else
    k_sample<E><<<a.N, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_sample(const SampleCall& a, hipStream_t s) {
  switch (a.dtype) {
    case RPD_DTYPE_BF16: sample_keys<Bf16>(a, s); break;
    case RPD_DTYPE_F16: sample_keys<F16>(a, s); break;
    default: k_sample<F32><<<a.N, kThreads, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace rpd
