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

struct Shared {
  Bins all, part;
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
  while (lo < hi) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __builtin_clz(span), shift = max(0, bits - 11);   // span >> shift < 2048
    __syncthreads();
    clear(s.part);
    __syncthreads();
    each<E>(row, V, [&](float z, int) {
      const uint32_t k = key_of(z);
      if (k >= lo && k <= hi) {
        const int i = (int)((hi - k) >> shift);
        atomicAdd(&s.part.n[i], 1u);
        atomicAdd(&s.part.mass[i], Weigh::mass(w.bins_below(z), b));
      }
    });
    __syncthreads();
    scan<false>(s.part, unit, s);
    const uint32_t i = (uint32_t)choose(s.part, q, n, m, s);
    count = s.part.n[i];
    hi -= i << shift;
    const uint32_t width = (1u << shift) - 1;
    lo = hi - lo > width ? hi - width : lo;
  }
  Place p;
  p.key = hi;
  p.n = n;
  p.eq = count;
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

template <class E>
__global__ __launch_bounds__(kThreads) void k_sample(SampleCall a) {
  __shared__ Shared s;
  const int n = blockIdx.x, t = threadIdx.x, lane = t & 63, wid = t >> 6, V = a.V;
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
  if (lane == 0) s.wave_top[wid] = top;
  if (lane == 0) s.wave_bad[wid] = 0;
  if (__any(bad) && lane == 0) s.wave_bad[wid] = 1;
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

}  // namespace

hipError_t launch_sample(const SampleCall& a, hipStream_t s) {
  switch (a.dtype) {
    case RPD_DTYPE_BF16: k_sample<Bf16><<<a.N, kThreads, 0, s>>>(a); break;
    case RPD_DTYPE_F16: k_sample<F16><<<a.N, kThreads, 0, s>>>(a); break;
    default: k_sample<F32><<<a.N, kThreads, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace rpd
