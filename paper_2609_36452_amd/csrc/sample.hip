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
// fixed-point sums relative to their bin's top (2^-42 of it, 64 bits): exact,
// and the same in whatever order the atomics come.
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

// Bin and mass of a logit. With d the distance below the maximum in bins, the
// mass relative to the bin's top is e^(-frac(d) / 32), by its series.
struct Weigh {
  double m, k;   // maximum, bins per unit of logit
  __device__ __forceinline__ Weigh(float top, float scale) : m((double)top), k((double)scale * kPerNat) {}
  __device__ __forceinline__ double bins_below(float z) const { return (m - (double)z) * k; }
  __device__ __forceinline__ int bin(float z) const {
    const double d = bins_below(z);
    return d < (double)kFar ? (int)d : kFar;
  }
  // fixed-point mass of a logit that is d bins below the maximum, in bin b
  static __device__ __forceinline__ unsigned long long mass(double d, int b) {
    if (b == kFar) return 0;
    const double x = ((double)b - d) * (1.0 / kPerNat);   // -1/32 .. 0
    double p = fma(x, 1.0 / 720, 1.0 / 120);
    p = fma(x, p, 1.0 / 24);
    p = fma(x, p, 1.0 / 6);
    p = fma(x, p, 0.5);
    p = fma(x, p, 1.0);
    p = fma(x, p, 1.0);
    // 2^52 added: the integer nearest to p 2^42 is the sum's low bits
    return (unsigned long long)__double_as_longlong(fma(p, kUnit, 4503599627370496.0)) & 0xfffffffffffffull;
  }
  static __device__ __forceinline__ double unit(int b) { return b == kFar ? 0.0 : exp(-(double)b / kPerNat) / kUnit; }
};

struct Bins {
  uint32_t n[kBins];               // tokens
  unsigned long long mass[kBins];
  uint32_t n_upto[kBins];          // and up to the bin's end
  double m_upto[kBins];
};

constexpr int kListed = 4096;   // tokens of a bin that are taken out of the row

struct Shared {
  Bins all, part;
  uint32_t list_key[kListed];
  int list_index[kListed];
  uint32_t listed;
  int list_bin;                    // whose tokens the list holds, or -1
  uint32_t wave_n[kWaves];
  double wave_m[kWaves];
  float wave_top[kWaves];
  int wave_bad[kWaves];
  uint32_t wave_in[kWaves];
  int found, last;
  uint32_t lo, hi;
  uint32_t n, eq;
  double m;
  int token;
  uint32_t slab[64];
};

// eight entries at a time of the row, f(value, index), -inf left out by the caller
template <class E, class F>
__device__ __forceinline__ void each(const typename E::t* row, int V, F f) {
  constexpr int kFlight = 4;
  for (int i0 = 8 * threadIdx.x; i0 < V; i0 += kFlight * 8 * kThreads) {
    Eight<E> v[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (i0 + u * 8 * kThreads < V) load_eight<E>(row, i0 + u * 8 * kThreads, V, v[u]);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int i = i0 + u * 8 * kThreads;
      if (i < V) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f(v[u].at(e) + 0.f, i + e);   // (past the end: -inf)
      }
    }
  }
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
  uint32_t sn = n[0] + n[1];
  double sm = m[0] + m[1];
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t on = __shfl_up(sn, k);
    const double om = __shfl_up(sm, k);
    sn += lane >= k ? on : 0;
    sm += lane >= k ? om : 0.0;
  }
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
// The token found: the `at`-th (by index) of `eq` tokens of the logit `key`, before which lie n tokens of mass m; each has mass w.
struct Place {
  uint32_t key, n, eq, at;
  int bin;
  double m, w;
  __device__ __forceinline__ uint32_t rank() const { return n + at; }
  __device__ __forceinline__ double upto() const { return m + (double)(at + 1) * w; }
};

// the bin in which the bound falls, with what lies before it (added to n, m)
__device__ __forceinline__ int choose(const Bins& b, const Bound& q, uint32_t& n, double& m, Shared& s) {
  if (threadIdx.x == 0) {
    s.found = kBins;
    s.last = -1;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = 2 * threadIdx.x + j;
    if (b.n[i] == 0) continue;
    const double upto = m + b.m_upto[i];
    const bool past = q.by_rank ? n + b.n_upto[i] > q.rank : q.reach ? upto >= q.mass : upto > q.mass;
    if (past) atomicMin(&s.found, i);
    else atomicMax(&s.last, i);
  }
  __syncthreads();
  const int i = s.found < kBins ? s.found : s.last;   // by rounding alone: the last that holds anything
  const uint32_t before = b.n_upto[i] - b.n[i];
  const double mass_before = before == 0 ? 0.0 : b.m_upto[max(i - 1, 0)];
  n += before;
  m += mass_before;
  __syncthreads();
  return i;
}

template <class E>
__device__ Place find(const typename E::t* row, int V, const Weigh& w, uint32_t top, const Bound& q, Shared& s) {
  uint32_t n = 0;
  double m = 0.0;
  const int b = choose(s.all, q, n, m, s);
  const double unit = Weigh::unit(b);
  uint32_t count = s.all.n[b];
  // The bin's logits are an interval: the first two waves find its ends, 64 steps at once. The bin falls as the key rises.
  {
    const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wid < 2) {
      // wave 0: the largest key of a bin >= b; wave 1: the smallest key of a bin <= b
      uint32_t lo = key_of(-3.402823466e38f), hi = top;   // bin(hi) = 0
      if (wid == 0) {
        while (lo < hi) {   // bin(lo) >= b, the answer in lo .. hi
          const uint32_t step = (hi - lo) / 64 + 1;
          const uint32_t k = lo + (uint32_t)(lane + 1) * step;
          const bool ok = k <= hi && k > lo && w.bin(value_of(k)) >= b;
          const int c = __popcll(__ballot(ok));   // the first c hold
          lo += c * step;
          hi = c == 64 ? hi : min(hi, lo + step - 1);
        }
        if (lane == 0) s.hi = lo;
      } else {
        while (lo < hi) {   // bin(hi) <= b
          const uint32_t step = (hi - lo) / 64 + 1;
          const uint32_t k = hi - (uint32_t)(lane + 1) * step;
          const bool ok = k >= lo && k < hi && w.bin(value_of(k)) <= b;
          const int c = __popcll(__ballot(ok));
          hi -= c * step;
          lo = c == 64 ? lo : hi - lo >= step ? hi - step + 1 : lo;
        }
        if (lane == 0) s.lo = hi;
      }
    }
    __syncthreads();
  }
  uint32_t lo = s.lo, hi = s.hi;
  const bool listed = count <= kListed;
  if (listed && s.list_bin != b) {
    __syncthreads();
    if (threadIdx.x == 0) {
      s.listed = 0;
      s.list_bin = b;
    }
    __syncthreads();
    each<E>(row, V, [&](float z, int i) {
      const uint32_t k = key_of(z);
      if (k >= lo && k <= hi) {
        const uint32_t at = atomicAdd(&s.listed, 1u);
        s.list_key[at] = k;
        s.list_index[at] = i;
      }
    });
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
        atomicAdd(&s.part.mass[i], Weigh::mass(w.bins_below(value_of(k)), b));
      }
    };
    if (listed) {
      for (uint32_t i = threadIdx.x; i < s.listed; i += kThreads) add(s.list_key[i]);
    } else {
      each<E>(row, V, [&](float z, int) { add(key_of(z)); });
    }
    __syncthreads();
    scan<false>(s.part, unit, s);
    const uint32_t i = (uint32_t)choose(s.part, q, n, m, s);
    count = s.part.n[i];
    hi -= i << shift;
    const uint32_t width = (1u << shift) - 1;
    lo = hi - lo > width ? hi - width : lo;
  }
  __syncthreads();
  Place p;
  p.key = hi;
  p.n = n;
  p.eq = count;
  p.bin = b;
  p.m = m;
  const float z = value_of(hi);
  p.w = (double)Weigh::mass(w.bins_below(z), b) * unit;
  if (q.by_rank) {
    p.at = min(q.rank - n, count - 1);
  } else {
    // the lowest i with m + (i + 1) w past the bound
    auto past = [&](double i) { return q.reach ? m + (i + 1.0) * p.w >= q.mass : m + (i + 1.0) * p.w > q.mass; };
    double i = p.w > 0.0 ? floor((q.mass - m) / p.w) : 0.0;
    i = fmin(fmax(i, 0.0), (double)(count - 1));
    while (i > 0.0 && past(i - 1.0)) i -= 1.0;
    while (i < (double)(count - 1) && !past(i)) i += 1.0;
    p.at = (uint32_t)i;
  }
  return p;
}

// the index of the at-th token (by index) of the logit `key`
template <class E>
__device__ int index_of(const typename E::t* row, int V, const Place& p, Shared& s) {
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6;
  __syncthreads();
  if (t < 64) s.slab[t] = 0;
  if (t == 0) s.token = -1;
  __syncthreads();
  if (s.list_bin == p.bin && p.eq <= 64) {
    for (uint32_t i = t; i < s.listed; i += kThreads) {
      if (s.list_key[i] != p.key) continue;
      uint32_t before = 0;
      for (uint32_t j = 0; p.eq > 1 && j < s.listed; ++j)
        before += s.list_key[j] == p.key && s.list_index[j] < s.list_index[i];
      if (before == p.at) s.token = s.list_index[i];
    }
    __syncthreads();
    return s.token;
  }
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
__device__ __noinline__ void sample_row(const SampleCall a, int n, Shared& s) {
  const int t = threadIdx.x, lane = t & 63, wid = t >> 6, V = a.V;
  const typename E::t* row = static_cast<const typename E::t*>(a.logits) + n * a.stride;
  typename E::t* out = a.filtered ? static_cast<typename E::t*>(a.filtered) + n * a.filtered_stride : nullptr;
  const float scale = a.scales ? a.scales[n] : a.scale;
  const int top_k = a.top_ks ? a.top_ks[n] : a.top_k;
  const float top_p = a.top_ps ? a.top_ps[n] : a.top_p, min_p = a.min_ps ? a.min_ps[n] : a.min_p;

  // the maximum; NaN, and +inf, leave no distribution
  float top = -INFINITY;
  bool bad = false;
  each<E>(row, V, [&](float z, int) {
    top = fmaxf(top, z);
    bad |= z != z;
  });
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
  const bool any_bad = __any(bad);
  if (lane == 0) {
    s.wave_top[wid] = top;
    s.wave_bad[wid] = any_bad;
  }
  if (t == 0) s.list_bin = -1;
  clear(s.all);
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    top = fmaxf(top, s.wave_top[w]);
    bad |= s.wave_bad[w] != 0;
  }
  const float sc = scale == 0.f ? 1.f : scale;
  if (bad || !(fabsf(top) < INFINITY) || !(sc > 0.f && sc < INFINITY)) {
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
  const bool least = min_p > 0.f;
  const double limit = least ? -log(fmin((double)min_p, 1.0)) * kPerNat : 0.0;
  uint32_t inside = 0;
  each<E>(row, V, [&](float z, int) {
    if (z > -INFINITY) {
      const double d = w.bins_below(z);
      const int b = d < (double)kFar ? (int)d : kFar;
      atomicAdd(&s.all.n[b], 1u);
      if (b != kFar) atomicAdd(&s.all.mass[b], Weigh::mass(d, b));
      inside += d <= limit;
    }
  });
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) inside += __shfl_xor(inside, k);
  if (lane == 0) s.wave_in[wid] = inside;
  __syncthreads();
  inside = 0;
  for (int v = 0; v < kWaves; ++v) inside += s.wave_in[v];
  scan<true>(s.all, 0.0, s);

  const uint32_t key_top = key_of(top);
  uint32_t kept = s.all.n_upto[kBins - 1];
  double mass = s.all.m_upto[kBins - 1];
  Place cut{};
  bool is_cut = false;
  if (top_k > 0 && (uint32_t)top_k < kept) {
    cut = find<E>(row, V, w, key_top, Bound{true, false, (uint32_t)top_k - 1, 0.0}, s);
    is_cut = true;
    kept = top_k;
    mass = cut.upto();
  }
  if (top_p < 1.f) {
    const Place p = find<E>(row, V, w, key_top, Bound{false, true, 0, fmax((double)top_p, 0.0) * mass}, s);
    if (p.rank() + 1 < kept) {
      cut = p;
      is_cut = true;
      kept = p.rank() + 1;
      mass = p.upto();
    }
  }
  if (least && inside < kept) {
    cut = find<E>(row, V, w, key_top, Bound{true, false, inside - 1, 0.0}, s);
    is_cut = true;
    kept = inside;
    mass = cut.upto();
  }
  Place p = find<E>(row, V, w, key_top, Bound{false, false, 0, (double)a.r[n] * mass}, s);
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
    if (i >= V) return;
    const uint32_t k = key_of(z);
    out[i] = k > key || (k == key && i <= last) ? row[i] : E::to(-INFINITY);
  });
}

template <class E>
__global__ __launch_bounds__(kThreads) void k_sample(SampleCall a) {
  __shared__ Shared s;
  sample_row<E>(a, blockIdx.x, s);
}

// ------------------------------------------------- 16-bit logits, held in registers --
//
// A row of up to 163840 logits of 16 bits fits a workgroup's registers, and a
// table with a 16-bit count for each of the 65536 values fits its LDS. So the
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
  const uint32_t sign = (w >> 15) & 0x10001u;
  return w ^ (0x7fff7fffu - sign * 0x7fffu);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct KeyBound {
  bool by_rank, reach;
  uint32_t rank;
  double mass;
};
struct KeyPlace {   // as Place, with a slot in place of the key
  uint32_t slot, n, eq, at;
  double m, w;
  __device__ __forceinline__ uint32_t rank() const { return n + at; }
  __device__ __forceinline__ double upto() const { return m + (double)(at + 1) * w; }
};

struct Keys {
  uint32_t count[32768];   // two values a word
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
};

// By the first wave: the token at which a bound is passed.
template <class E>
__device__ __forceinline__ KeyPlace find_key(const Keys& s, const Weigh& w, const KeyBound& q) {
  const int lane = threadIdx.x & 63;
  // the block: each lane looks at 16 in a row
  int first = kThreads, last = -1;
#pragma unroll 4
  for (int j = 15; j >= 0; --j) {
    const int b = lane * 16 + j;
    const uint32_t upto = s.n_upto[b], n = upto - (b ? s.n_upto[b - 1] : 0);
    const double m = s.m_upto[b];
    const bool past = q.by_rank ? upto > q.rank : q.reach ? m >= q.mass : m > q.mass;
    if (n > 0 && past) first = b;
    if (n > 0) last = max(last, b);
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    first = min(first, __shfl_xor(first, k));
    last = max(last, __shfl_xor(last, k));
  }
  const int b = first < kThreads ? first : last;   // by rounding alone: the last that holds anything
  const uint32_t n0 = b ? s.n_upto[b - 1] : 0;
  const double m0 = b ? s.m_upto[b - 1] : 0.0;
  // the value, a lane each
  const uint32_t slot = b * 64 + lane, word = s.count[slot >> 1], c = slot & 1 ? word >> 16 : word & 0xffff;
  const double e = c ? exp(w.bins_below(slot_value<E>(slot)) * (-1.0 / kPerNat)) : 0.0;
  uint32_t n = c;
  double m = c * e;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t on = __shfl_up(n, k);
    const double om = __shfl_up(m, k);
    n += lane >= k ? on : 0;
    m += lane >= k ? om : 0.0;
  }
  const bool past = c > 0 && (q.by_rank ? n0 + n > q.rank : q.reach ? m0 + m >= q.mass : m0 + m > q.mass);
  const unsigned long long hits = __ballot(past), some = __ballot(c > 0);
  const int at = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(some);
  const uint32_t before = __shfl_up(n, 1);
  const double m_before = __shfl_up(m, 1);
  KeyPlace p;
  p.slot = b * 64 + at;
  p.eq = __shfl(c, at);
  p.n = n0 + (at ? __shfl(before, at) : 0);
  p.m = m0 + (at ? __shfl(m_before, at) : 0.0);
  p.w = __shfl(e, at);
  if (q.by_rank) {
    p.at = min(q.rank - p.n, p.eq - 1);
  } else {
    auto over = [&](double i) { return q.reach ? p.m + (i + 1.0) * p.w >= q.mass : p.m + (i + 1.0) * p.w > q.mass; };
    double i = p.w > 0.0 ? floor((q.mass - p.m) / p.w) : 0.0;
    i = fmin(fmax(i, 0.0), (double)(p.eq - 1));
    while (i > 0.0 && over(i - 1.0)) i -= 1.0;
    while (i < (double)(p.eq - 1) && !over(i)) i += 1.0;
    p.at = (uint32_t)i;
  }
  return p;
}

template <class E, int NV>
__global__ __launch_bounds__(kThreads) void k_sample_keys(SampleCall a) {
  constexpr size_t kBytes = sizeof(Keys) > sizeof(Shared) ? sizeof(Keys) : sizeof(Shared);
  __shared__ __attribute__((aligned(16))) unsigned char lds[kBytes];
  Keys& s = *reinterpret_cast<Keys*>(lds);
  const int n = blockIdx.x, t = threadIdx.x, lane = t & 63, wid = t >> 6, V = a.V;
  const typename E::t* row = static_cast<const typename E::t*>(a.logits) + n * a.stride;
  const float scale = a.scales ? a.scales[n] : a.scale;
  const int top_k = a.top_ks ? a.top_ks[n] : a.top_k;
  const float top_p = a.top_ps ? a.top_ps[n] : a.top_p, min_p = a.min_ps ? a.min_ps[n] : a.min_p;

  uint32_t v[NV][4];   // vector j holds tokens 8 (t + 1024 j) .. of the row
  const int steps = (V + 8 * kThreads - 1) / (8 * kThreads);
  Eight<E> end_of_row;
  constexpr uint32_t kLows = Slots<E>::low * 0x10001u;
  end_of_row.v = u32x4{kLows, kLows, kLows, kLows};
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    u32x4 x = {kLows, kLows, kLows, kLows};
    if (j < steps - 1) x = reinterpret_cast<const Any16*>(row + 8 * (t + j * kThreads))->v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[j][e] = x[e];
  }
  if (8 * (t + (steps - 1) * kThreads) < V) load_eight<E>(row, 8 * (t + (steps - 1) * kThreads), V, end_of_row);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[j][e] = j == steps - 1 ? end_of_row.v[e] : v[j][e];
  for (int i = t; i < 8192; i += kThreads) reinterpret_cast<u32x4*>(s.count)[i] = u32x4{0u, 0u, 0u, 0u};
  if (t < 64) s.slab[t] = 0;
  if (t == 0) {
    s.give_up = 0;
    s.token = -1;
  }
  u16x2 lo = {0xffff, 0xffff}, hi = {0, 0};
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[j][e] = slots_of(v[j][e]);
      asm("" : "+v"(v[j][e]));   // kept in place of what it came from
      lo = __builtin_elementwise_min(lo, __builtin_bit_cast(u16x2, v[j][e]));
      hi = __builtin_elementwise_max(hi, __builtin_bit_cast(u16x2, v[j][e]));
    }
  }
  uint32_t first = min((uint32_t)lo.x, (uint32_t)lo.y), last = max((uint32_t)hi.x, (uint32_t)hi.y);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    first = min(first, (uint32_t)__shfl_xor((int)first, k));
    last = max(last, (uint32_t)__shfl_xor((int)last, k));
  }
  if (lane == 0) {
    s.wave_lo[wid] = first;
    s.wave_hi[wid] = last;
  }
  __syncthreads();
  for (int k = 0; k < kWaves; ++k) {
    first = min(first, s.wave_lo[k]);
    last = max(last, s.wave_hi[k]);
  }
  if (first == kMinusZero) first = kZero;
  const float top = slot_value<E>(first), sc = scale == 0.f ? 1.f : scale;
  // NaN (on either side) or +inf in the row, nothing but -inf, or no temperature
  if (last > Slots<E>::low || first >= Slots<E>::low || !(fabsf(top) < INFINITY) || !(sc > 0.f && sc < INFINITY)) {
    __syncthreads();
    sample_row<E>(a, n, *reinterpret_cast<Shared*>(lds));
    return;
  }
  const Weigh w(top, sc);
  const bool least = min_p > 0.f;
  const double limit = least ? -log(fmin((double)min_p, 1.0)) * kPerNat : 0.0;
  // slots beyond `end` are not counted: 64 nats below; of min_p alone, what it leaves out (`limit` and a little more)
  const bool min_alone = least && top_k <= 0 && !(top_p < 1.f);
  const double reach_bins = min_alone ? fmin(limit + 1.0, 64.0 * kPerNat) : 64.0 * kPerNat;
  const uint32_t end = min(slot_of<E>((float)((double)top - reach_bins / ((double)sc * kPerNat))), Slots<E>::low - 1);
  uint32_t infs = 0, seen = 0;   // seen: what was counted
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (j < steps) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = v[j][e], x0 = x & 0xffff, x1 = x >> 16;
        if (x0 <= end) atomicAdd(&s.count[x0 >> 1], x0 & 1 ? 0x10000u : 1u);
        if (x1 <= end) atomicAdd(&s.count[x1 >> 1], x1 & 1 ? 0x10000u : 1u);
        infs += (x0 == Slots<E>::low) + (x1 == Slots<E>::low);
        seen += (x0 <= end) + (x1 <= end);
      }
    }
    __builtin_amdgcn_sched_barrier(0);   // one vector at a time: the row takes most of the registers
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    infs += __shfl_xor(infs, k);
    seen += __shfl_xor(seen, k);
  }
  if (lane == 0) {
    s.wave_n[wid] = infs;
    s.wave_hi[wid] = seen;
  }
  __syncthreads();
  infs = seen = 0;
  for (int k = 0; k < kWaves; ++k) {
    infs += s.wave_n[k];
    seen += s.wave_hi[k];
  }
  const uint32_t finite = (uint32_t)(steps * 8 * kThreads) - infs;   // (what is past the row's end is -inf as well)
  if (t == 0) {   // the two zeros are equal
    const uint32_t minus = s.count[kMinusZero >> 1] & 0xffff;
    if (minus) {
      if ((s.count[kZero >> 1] >> 16) + minus > 0xffff) s.give_up = 1;
      s.count[kZero >> 1] += minus << 16;
      s.count[kMinusZero >> 1] -= minus;
    }
  }
  __syncthreads();
  // the block of 64 values: z_i = z_0 - i u from the maximum's slot on, so the masses are e_0 rho^i
  uint32_t bn = 0;
  double bm = 0.0;
  {
    const u32x4* p = reinterpret_cast<const u32x4*>(&s.count[t * 32]);
    uint32_t any = 0;
#pragma unroll 4
    for (int j = 0; j < 8; ++j) {
      const u32x4 c = p[(j + t) & 7];   // lanes 128 bytes apart: spread over the banks
      any |= c[0] | c[1] | c[2] | c[3];
    }
    if (any) {
      const uint32_t start = t * 64;
      const int i0 = first > start ? (int)(first - start) : 0;
      const float z0 = slot_value<E>(start + i0), u = slot_value<E>(start) - slot_value<E>(start + 1);
      const double e0 = exp(w.bins_below(z0) * (-1.0 / kPerNat)), rho = exp(-(double)u * w.k * (1.0 / kPerNat));
#pragma unroll 2
      for (int i = 31; i >= 0; --i) {
        const uint32_t x = s.count[t * 32 + i];
        if (2 * i + 1 >= i0) {
          bm = fma(bm, rho, (double)(x >> 16));
          if (2 * i >= i0) bm = fma(bm, rho, (double)(x & 0xffff));
        }
        bn += (x & 0xffff) + (x >> 16);
      }
      bm *= e0;
    }
  }
  uint32_t un = bn;
  double um = bm;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t on = __shfl_up(un, k);
    const double om = __shfl_up(um, k);
    un += lane >= k ? on : 0;
    um += lane >= k ? om : 0.0;
  }
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
  const bool low = least && limit > 63.0 * kPerNat;
  if (seen != counted || s.give_up || far || low) {
    __syncthreads();
    sample_row<E>(a, n, *reinterpret_cast<Shared*>(lds));
    return;
  }
  if (wid == 0) {
    uint32_t kept = finite;
    double mass = s.m_upto[kThreads - 1];
    KeyPlace cut{};
    bool is_cut = false;
    if (top_k > 0 && (uint32_t)top_k < kept) {
      cut = find_key<E>(s, w, KeyBound{true, false, (uint32_t)top_k - 1, 0.0});
      is_cut = true;
      kept = top_k;
      mass = cut.upto();
    }
    if (top_p < 1.f) {
      const KeyPlace p = find_key<E>(s, w, KeyBound{false, true, 0, fmax((double)top_p, 0.0) * mass});
      if (p.rank() + 1 < kept) {
        cut = p;
        is_cut = true;
        kept = p.rank() + 1;
        mass = p.upto();
      }
    }
    if (least) {
      // the blocks whose first value min_p leaves, then the values of the last of them
      int b = 0;
#pragma unroll 2
      for (int j = 0; j < 16; ++j) {
        const int k = lane * 16 + j;
        const uint32_t x = min(max((uint32_t)k * 64, first), Slots<E>::low - 1);
        if (w.bins_below(slot_value<E>(x)) <= limit) b = k;
      }
#pragma unroll
      for (int k = 32; k >= 1; k >>= 1) b = max(b, __shfl_xor(b, k));
      const uint32_t slot = b * 64 + lane, word = s.count[slot >> 1], c = slot & 1 ? word >> 16 : word & 0xffff;
      uint32_t in = c && w.bins_below(slot_value<E>(slot)) <= limit ? c : 0;
#pragma unroll
      for (int k = 32; k >= 1; k >>= 1) in += __shfl_xor(in, k);
      in += b ? s.n_upto[b - 1] : 0;
      if (in < kept) {
        cut = find_key<E>(s, w, KeyBound{true, false, in - 1, 0.0});
        is_cut = true;
        kept = in;
        mass = cut.upto();
      }
    }
    KeyPlace p = find_key<E>(s, w, KeyBound{false, false, 0, (double)a.r[n] * mass});
    if (is_cut && p.rank() > cut.rank()) p = cut;   // by rounding alone
    if (lane == 0) {
      s.pick = p;
      s.cut = cut;
      s.is_cut = is_cut;
      if (a.prob) a.prob[n] = (float)(p.w / mass);
      if (a.kept) a.kept[n] = (int)kept;
    }
  }
  __syncthreads();
  // the index of the at-th token of a slot: in order of j, then of the threads, then inside the vector
  auto index_of = [&](const KeyPlace& p) __attribute__((always_inline)) {
    auto same = [&](uint32_t x) __attribute__((always_inline)) { return x == p.slot || (p.slot == kZero && x == kMinusZero); };
    __syncthreads();
    if (t == 0) s.token = -1;
    if (t < 64) s.slab[t] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j >= steps) continue;
      uint32_t c = 0;
      int at = 0;
#pragma unroll
      for (int e = 3; e >= 0; --e) {
        const bool h = same(v[j][e] >> 16), l = same(v[j][e] & 0xffff);
        at = l ? 2 * e : h ? 2 * e + 1 : at;
        c += h + l;
      }
      if (c) {
        if (p.eq == 1) s.token = 8 * (t + j * kThreads) + at;
        else atomicAdd(&s.slab[j], c);
      }
    }
    __syncthreads();
    if (p.eq > 1) {
      uint32_t before = 0;
      int slab = 0;
      for (; slab < NV - 1 && before + s.slab[slab] <= p.at; ++slab) before += s.slab[slab];
      uint32_t c = 0, mask = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (j == slab) {
#pragma unroll
          for (int e = 0; e < 8; ++e) mask |= (uint32_t)same(e & 1 ? v[j][e >> 1] >> 16 : v[j][e >> 1] & 0xffff) << e;
        }
      c = __popc(mask);
      uint32_t upto = c;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const uint32_t o = __shfl_up(upto, k);
        upto += lane >= k ? o : 0;
      }
      if (lane == 63) s.wave_n[wid] = upto;
      __syncthreads();
      for (int k = 0; k < wid; ++k) before += s.wave_n[k];
      before += upto - c;
      if (p.at >= before && p.at < before + c) {
        for (uint32_t i = before; i < p.at; ++i) mask &= mask - 1;
        s.token = 8 * (t + slab * kThreads) + __builtin_ctz(mask);
      }
      __syncthreads();
    }
    return s.token;
  };
  const int token = index_of(s.pick);
  if (t == 0) a.token[n] = token;
  if (!a.filtered) return;
  typename E::t* out = static_cast<typename E::t*>(a.filtered) + n * a.filtered_stride;
  // what comes before the cut's slot stays, and of its tokens those up to the last kept one
  const KeyPlace cut = s.cut;
  const bool is_cut = s.is_cut;
  uint32_t slot = is_cut ? cut.slot : Slots<E>::low;
  int until = V;
  if (is_cut && cut.at + 1 < cut.eq) until = index_of(cut);
  if (slot == kZero) slot = kMinusZero;
  const uint32_t after = slot, tie = is_cut && cut.slot == kZero ? kZero : slot;   // ties: tie .. after
  const uint32_t gone = E::to(-INFINITY);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i0 = 8 * (t + j * kThreads);
    if (j >= steps || i0 >= V) continue;
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = v[j][e], x0 = x & 0xffff, x1 = x >> 16;
      const bool k0 = x0 < tie || (x0 <= after && i0 + 2 * e <= until), k1 = x1 < tie || (x1 <= after && i0 + 2 * e + 1 <= until);
      const uint32_t b = slots_of(x);   // its own inverse on the sign's halves
      o[e] = (k0 ? b & 0xffff : gone) | (k1 ? b & 0xffff0000u : gone << 16);
    }
    if (i0 + 8 <= V) {
      reinterpret_cast<Any16*>(out + i0)->v = o;
    } else {
      for (int e = 0; i0 + e < V; ++e) out[i0 + e] = (typename E::t)(o[e >> 1] >> (16 * (e & 1)));
    }
  }
}

template <class E>
void sample_keys(const SampleCall& a, hipStream_t s) {
  constexpr int kStep = 8 * kThreads;
  if (a.V <= 4 * kStep)
    k_sample_keys<E, 4><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 10 * kStep)
    k_sample_keys<E, 10><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 16 * kStep)
    k_sample_keys<E, 16><<<a.N, kThreads, 0, s>>>(a);
  else if (a.V <= 20 * kStep)
    k_sample_keys<E, 20><<<a.N, kThreads, 0, s>>>(a);
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
