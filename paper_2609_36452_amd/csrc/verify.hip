// Verification of drafted tokens against a target's logits, from given random
// numbers.
//
//   p_t = softmax(target_scale z_t), q_t = softmax(draft_scale y_t)
//   a_t = min(1, p_t(x_t) / q_t(x_t)); token t is accepted while u_t < a_t
//   after n accepted: w = max(0, p_n - q_n) if token n was turned down (p_n
//   where that is empty), p_n if the draft ended; the next token is the lowest
//   v with w_0 + .. + w_v > r sum w
//
// Bound: one read of the rows, and for the small calls the latency of the
// launches. The steps:
//   k_verify_stats   maximum and sum of a part of a row, every row at once
//   k_verify_decide  a sequence's acceptance probabilities, n, and the row that
//                    the further token is drawn from (many rows; of few rows
//                    every workgroup of k_verify_parts does that for itself)
//   k_verify_totals  float64 sums of that row (after float32 statistics)
//   k_verify_parts   sums of max(0, p - q), and of p, over parts of that row
//   k_verify_token   the part that r falls in, then the token in it
// A launch that waits for the one before it takes 4 us however little it does:
// 5 target and 4 draft rows of 126464 bf16 take 15.2 us in three launches, and
// the decision as a fourth 2.4 us more. (A draw by the last workgroup to finish
// its part needs no launch either, but the release and acquire cost 62 parts
// as much as it, and 32 x 38 parts 14 us more.)
// The draw is float64, exponentials included: the token's border lies among up
// to V cumulative sums a few 1e-6 apart, and in float32 a draw in a hundred of
// a flat row would fall on the neighbour of the right token. Few rows take
// their statistics in float64 as well, which saves two launches; many do not
// (a float64 exponential is 12 double operations at half the rate of single
// ones: 288 target and 130 draft rows of 152064 bf16 take 39 us, 18 in float32).
#include <cstdint>

#include "logit_rows.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr double k32PerLn2 = 46.166241308446828384;   // 32 / ln 2

// e^(scale z - scale m) in float64, to about 1e-12: with z in units of 1/32
// octave, n the nearest whole one and f the rest, 2^(n >> 5) by the exponent,
// 2^((n & 31) / 32) from a table of 32 (one entry per pair of LDS banks: no
// conflicts) and e^(f ln 2 / 32) by its series to the fourth power.
struct Exp64 {
  static constexpr double kLow = -31800.0;   // 1/32 octaves below which it is 0 (the exponent stays a normal one)
  double k, m;
  const double* table;
  __device__ __forceinline__ Exp64(float top, float scale, const double* t)
      : k((double)scale * k32PerLn2), m(top == -INFINITY ? 0.0 : (double)top), table(t) {}
  // the difference first: rows far from 0 lose nothing
  __device__ __forceinline__ double octaves(float z) const { return ((double)z - m) * k; }
  // t at least kLow
  __device__ __forceinline__ double power(double t) const {
    constexpr double u = 0.021660849392498290;   // ln 2 / 32
    constexpr double kShift = 6755399441055744.0;   // 1.5 * 2^52: the sum's low word is the nearest integer
    const double s = t + kShift, f = t - (s - kShift);
    double p = fma(f, u * u * u * u / 24, u * u * u / 6);
    p = fma(f, p, u * u / 2);
    p = fma(f, p, u);
    p = fma(f, p, 1.0);
    const int n = __double2loint(s);
    const double w = table[n & 31];
    return p * __hiloint2double(__double2hiint(w) + ((n >> 5) << 20), __double2loint(w));
  }
  __device__ __forceinline__ double operator()(float z) const {
    const double t = octaves(z);
    return t < kLow ? 0.0 : power(t);
  }
  // for sums: below kLow what is added is less than 1e-299 (NaN stays NaN)
  __device__ __forceinline__ double about(float z) const {
    const double t = octaves(z);
    return power(t < kLow ? kLow : t);
  }
};
// 2^(j / 32)
__device__ const double kPowers[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002,
};
__device__ __forceinline__ void fill_table(double* t) {
  if (threadIdx.x < 32) t[threadIdx.x] = kPowers[threadIdx.x];
}

template <class E>
__device__ __forceinline__ const typename E::t* target_row(const VerifyCall& a, int b, int t) {
  return static_cast<const typename E::t*>(a.target) + b * a.t_batch + t * a.t_row;
}
template <class E>
__device__ __forceinline__ const typename E::t* draft_row(const VerifyCall& a, int b, int t) {
  return static_cast<const typename E::t*>(a.draft) + b * a.d_batch + t * a.d_row;
}
__device__ __forceinline__ int draft_len(const VerifyCall& a, int b) {
  return a.len ? min(max(a.len[b], 0), a.T) : a.T;
}

// rows: the target's B (T + 1), then the draft's B T
enum Stats { kGreedy, kDouble, kSingle };   // maximum and its lowest index; maximum and sum in float64 or float32
template <class E, Stats KIND>
__global__ __launch_bounds__(kThreads) void k_verify_stats(VerifyCall a) {
  const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits;
  const bool is_draft = row >= a.B * (a.T + 1);
  const int rr = is_draft ? row - a.B * (a.T + 1) : row, per = is_draft ? a.T : a.T + 1;
  const int b = rr / per, t = rr - b * per;
  if (is_draft ? t >= draft_len(a, b) : t > draft_len(a, b)) return;   // rows behind the draft are not read
  const typename E::t* p = is_draft ? draft_row<E>(a, b, t) : target_row<E>(a, b, t);
  const int lo = split * a.chunk, hi = min(a.V, lo + a.chunk);
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  __shared__ float s_max[kWaves];
  __shared__ int s_idx[kWaves];
  __shared__ double s_sum[kWaves], s_table[32];
  // the part's first vectors are held, a longer part's others read again
  constexpr int kHeld = 4;
  Eight<E> held[kHeld];
  auto get = [&](int i, Eight<E>& v) { load_eight<E>(p, i, hi, v); };
  const int first = lo + 8 * threadIdx.x;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (first + j * 8 * kThreads < hi) get(first + j * 8 * kThreads, held[j]);
  if (KIND == kDouble) fill_table(s_table);
  float m = -INFINITY;
  int idx = INT_MAX;
  auto top = [&](int i, const Eight<E>& v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float z = v.at(e);
      if (KIND == kGreedy) idx = z > m ? i + e : idx;
      m = fmaxf(m, z);
    }
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (first + j * 8 * kThreads < hi) top(first + j * 8 * kThreads, held[j]);
  for (int i = first + kHeld * 8 * kThreads; i < hi; i += 8 * kThreads) {
    Eight<E> v;
    get(i, v);
    top(i, v);
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    const float om = __shfl_xor(m, k);
    if (KIND == kGreedy) {
      const int oi = __shfl_xor(idx, k);
      idx = om > m ? oi : om < m ? idx : min(idx, oi);
    }
    m = fmaxf(m, om);
  }
  if (lane == 0) {
    s_max[wid] = m;
    s_idx[wid] = idx;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    const float om = s_max[w];
    if (KIND == kGreedy) idx = om > m ? s_idx[w] : om < m ? idx : min(idx, s_idx[w]);
    m = fmaxf(m, om);
  }
  RowPart& out = a.stats[(long long)row * a.splits + split];
  if (KIND == kGreedy) {
    if (threadIdx.x == 0) out = RowPart{0.0, m, idx};
    return;
  }
  const float scale = is_draft ? a.draft_scale : a.target_scale, below = top_of(m);
  const Exp64 ex(m, scale, s_table);
  double sum = 0.0;
  float single = 0.f;
  auto add = [&](const Eight<E>& v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (KIND == kDouble)
        sum += ex.about(v.at(e));
      else
        single += exp_below(v.at(e), below, scale);
    }
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (first + j * 8 * kThreads < hi) add(held[j]);
  for (int i = first + kHeld * 8 * kThreads; i < hi; i += 8 * kThreads) {
    Eight<E> v;
    get(i, v);
    add(v);
  }
  if (KIND == kSingle) sum = single;
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) sum += __shfl_xor(sum, k);
  if (lane == 0) s_sum[wid] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWaves; ++w) sum += s_sum[w];
    // a part of nothing but -inf has no sum (one of NaN does not end here: its sum is NaN)
    out = RowPart{m == -INFINITY && sum == sum ? 0.0 : sum, m, 0};
  }
}

// a row's maximum and sum, by one wave in a fixed order
struct Row {
  float m;
  double S;
};
__device__ __forceinline__ Row row_stats(const VerifyCall& a, long long row, float scale, int lane,
                                         const double* table) {
  RowPart v{0.0, -INFINITY, 0};   // (at most 64 parts a row)
  if (lane < a.splits) v = a.stats[row * a.splits + lane];
  float m = v.m;
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  double S = v.m == -INFINITY ? v.S : v.S * Exp64(m, scale, table)(v.m);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) S += __shfl_xor(S, k);
  return Row{m, S};
}

// A sequence's acceptance probabilities, n and the rows that its further token is drawn from, by a workgroup, a wave a
// row in turn. A wave keeps the statistics of the first token it turns down (and of the row behind the draft, which
// ends it as well); the one with the first of all has the pick. Of several workgroups that do this for one sequence,
// one writes the results.
struct Decision {
  VerifyPick pick;
  int n;
};
template <class E, int WAVES>
__device__ __forceinline__ void decide(const VerifyCall& a, int b, bool write, Decision& s, double* table) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int len = draft_len(a, b);
  if (threadIdx.x == 0) s.n = len;
  fill_table(table);
  __syncthreads();
  const long long t0 = (long long)b * (a.T + 1), d0 = (long long)a.B * (a.T + 1) + (long long)b * a.T;
  int mine = INT_MAX;
  VerifyPick pick;
  for (int t = wid; t <= len; t += WAVES) {
    const bool drafted = t < len;
    const int x = drafted ? a.token[(long long)b * a.T + t] : -1;
    const float u = drafted ? a.u[(long long)b * a.T + t] : 0.f;
    const bool valid = x >= 0 && x < a.V;
    const float zp = valid ? E::one(target_row<E>(a, b, t) + x) : -INFINITY;
    const float zq = valid && a.draft ? E::one(draft_row<E>(a, b, t) + x) : 0.f;
    const Row p = row_stats(a, t0 + t, a.target_scale, lane, table);
    Row q{0.f, 1.0};
    if (a.draft && drafted) q = row_stats(a, d0 + t, a.draft_scale, lane, table);
    float acc = 0.f;
    if (drafted) {
      // one exponential of both distances: the quotient overflows only where it is far above 1
      double l = ((double)zp - (double)p.m) * (double)a.target_scale;
      if (a.draft) l -= ((double)zq - (double)q.m) * (double)a.draft_scale;
      const double quotient = exp(l) * (q.S / p.S);
      acc = !valid ? 0.f : quotient > 1.0 ? 1.f : (float)quotient;
      if (write && lane == 0) a.accept[(long long)b * a.T + t] = acc;
    }
    if (mine == INT_MAX && !(drafted && u < acc)) {
      mine = t;
      pick = VerifyPick{p.S, q.S, p.m, q.m, x, drafted};
      if (lane == 0) atomicMin(&s.n, t);
    }
  }
  if (write)
    for (int t = len + threadIdx.x; t < a.T; t += WAVES * 64) a.accept[(long long)b * a.T + t] = 0.f;
  __syncthreads();
  if (lane == 0 && mine == s.n) {
    s.pick = pick;
    if (write) a.n_accept[b] = mine;
  }
  __syncthreads();
}

constexpr int kDecideWaves = 8;
template <class E>
__global__ __launch_bounds__(kDecideWaves * 64) void k_verify_decide(VerifyCall a) {
  __shared__ Decision s;
  __shared__ double s_table[32];
  decide<E, kDecideWaves>(a, blockIdx.x, true, s, s_table);
  if (threadIdx.x == 0) a.picks[blockIdx.x] = s.pick;
}

// max(0, p - q) of a sequence whose token n was turned down
template <class E>
struct Rest {
  const typename E::t *p, *q;   // q NULL: 1 at x
  Exp64 ep, eq;
  double ip, iq;
  int x;
  __device__ __forceinline__ Rest(const VerifyCall& a, int b, int n, const VerifyPick& k, double sp, double sq,
                                  const double* table)
      : p(target_row<E>(a, b, n)), q(a.draft ? draft_row<E>(a, b, n) : nullptr), ep(k.mp, a.target_scale, table),
        eq(k.mq, a.draft_scale, table), ip(1.0 / sp), iq(1.0 / sq), x(k.x) {}
  __device__ __forceinline__ void fetch(int i, int V, bool down, Eight<E>& vp, Eight<E>& vq) const {
    load_eight<E>(p, i, V, vp);
    if (down && q) load_eight<E>(q, i, V, vq);
  }
  // p of the 8 entries from i on (0 past the row's end) and, of a token turned down, the rest
  __device__ __forceinline__ void eight(int i, bool down, const Eight<E>& vp, const Eight<E>& vq, double (&p8)[8],
                                        double (&w)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p8[e] = ep(vp.at(e)) * ip;
      w[e] = 0.0;
      if (!down) continue;
      if (q)
        w[e] = p8[e] - eq(vq.at(e)) * iq;
      else
        w[e] = i + e == x ? 0.0 : p8[e];
      w[e] = w[e] > 0.0 ? w[e] : 0.0;
    }
  }
};

// Vectors of a part that a thread has in flight: a part of 4096 entries is one round (rows of up to 262144; one vector
// at a time, two in turn, takes 2 us more over three passes of 32 pairs of rows of 152064).
constexpr int kFlight = 2;

// Float64 sums over parts of the sampled rows, where the statistics are float32.
template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_totals(VerifyCall a) {
  const int part = blockIdx.x % a.parts, b = blockIdx.x / a.parts, n = a.n_accept[b];
  const VerifyPick k = a.picks[b];
  __shared__ double s_sum[kWaves][2], s_table[32];
  fill_table(s_table);
  __syncthreads();
  const Exp64 ep(k.mp, a.target_scale, s_table), eq(k.mq, a.draft_scale, s_table);
  const typename E::t* p = target_row<E>(a, b, n);
  const typename E::t* q = a.draft && k.down ? draft_row<E>(a, b, n) : nullptr;
  const int hi = min(a.V, (part + 1) * a.part);
  double sum[2] = {0.0, 0.0};
  for (int i = part * a.part + 8 * threadIdx.x; i < hi; i += kFlight * 8 * kThreads) {
    Eight<E> vp[kFlight], vq[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int at = i + u * 8 * kThreads;
      if (at >= hi) continue;
      load_eight<E>(p, at, hi, vp[u]);
      if (q) load_eight<E>(q, at, hi, vq[u]);
    }
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      if (i + u * 8 * kThreads >= hi) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[0] += ep.about(vp[u].at(e));
      if (q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[1] += eq.about(vq[u].at(e));
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int j = 32; j >= 1; j >>= 1) sum[c] += __shfl_xor(sum[c], j);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6][c] = sum[c];
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    double t = 0.0;
    for (int w = 0; w < kWaves; ++w) t += s_sum[w][threadIdx.x];
    a.totals[((long long)threadIdx.x * a.B + b) * a.parts + part] = t;
  }
}

// the sums of the sampled rows, by each wave in a fixed order (NaN and an empty row end as in the statistics)
__device__ __forceinline__ void sampled_sums(const VerifyCall& a, int b, const VerifyPick& k, int lane, double& sp,
                                             double& sq) {
  double t[2] = {0.0, 0.0};
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane < a.parts) t[c] = a.totals[((long long)c * a.B + b) * a.parts + lane];   // (at most 64 parts)
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 32; j >= 1; j >>= 1) t[c] += __shfl_xor(t[c], j);
  if (k.mp > -INFINITY) sp = t[0];
  if (a.draft && k.down && k.mq > -INFINITY) sq = t[1];
}

// The parts of sum p and, where a token was turned down, of sum max(0, p - q).
// DECIDE: every workgroup decides for itself beforehand, with more waves for that.
template <class E, bool DECIDE>
__global__ __launch_bounds__(DECIDE ? kDecideWaves * 64 : kThreads) void k_verify_parts(VerifyCall a) {
  constexpr int W = DECIDE ? kDecideWaves : kWaves;
  const int part = blockIdx.x % a.parts, b = blockIdx.x / a.parts;
  __shared__ double s_sum[W][2], s_table[32];
  __shared__ Decision s;
  if (DECIDE) {
    decide<E, W>(a, b, part == 0, s, s_table);
    if (part == 0 && threadIdx.x == 0) a.picks[b] = s.pick;
  } else {
    if (threadIdx.x == 0) s = Decision{a.picks[b], a.n_accept[b]};
    fill_table(s_table);
    __syncthreads();
  }
  const VerifyPick k = s.pick;
  const int n = s.n;
  double sp = k.sp, sq = k.sq;
  if (!DECIDE) sampled_sums(a, b, k, threadIdx.x & 63, sp, sq);
  const Rest<E> rest(a, b, n, k, sp, sq, s_table);
  const int hi = min(a.V, (part + 1) * a.part);
  double sum[2] = {0.0, 0.0};
  for (int i = part * a.part + 8 * threadIdx.x; i < hi; i += kFlight * 8 * 64 * W) {
    Eight<E> vp[kFlight], vq[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)   // (a part ends at the row's end or at a whole vector)
      if (i + u * 8 * 64 * W < hi) rest.fetch(i + u * 8 * 64 * W, a.V, k.down, vp[u], vq[u]);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      if (i + u * 8 * 64 * W >= hi) continue;
      double p[8], w[8];
      rest.eight(i + u * 8 * 64 * W, k.down, vp[u], vq[u], p, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum[0] += p[e];
        sum[1] += w[e];
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int j = 32; j >= 1; j >>= 1) sum[c] += __shfl_xor(sum[c], j);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6][c] = sum[c];
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    double t = 0.0;
    for (int w = 0; w < W; ++w) t += s_sum[w][threadIdx.x];
    a.sums[((long long)threadIdx.x * a.B + b) * a.parts + part] = t;
  }
}

__device__ __forceinline__ double wave_scan(double v, int lane) {   // inclusive
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const double o = __shfl_up(v, k);
    v += lane >= k ? o : 0.0;
  }
  return v;
}

template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_token(VerifyCall a) {
  const int b = blockIdx.x, lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  // everything that does not depend on the part, at once (at most 64 parts, a lane each)
  const int n = a.n_accept[b];
  const VerifyPick k = a.picks[b];
  const float r = a.r[b];
  double weight[2] = {0.0, 0.0};   // of p, of the draft's rest
  if (lane < a.parts) {
    weight[0] = a.sums[(long long)b * a.parts + lane];
    weight[1] = a.sums[((long long)a.B + b) * a.parts + lane];
  }
  double sp = k.sp, sq = k.sq;
  if (a.totals) sampled_sums(a, b, k, lane, sp, sq);
  __shared__ double s_table[32], s_wave[kWaves];
  __shared__ int s_token, s_last;
  fill_table(s_table);
  if (threadIdx.x == 0) {
    s_token = INT_MAX;
    s_last = -1;
  }
  __syncthreads();
  // the part in which the running sum passes r of the whole (by rounding alone, the last that holds anything), by each
  // wave; of the draft's rest, or where there is none of the target's row
  bool use_rest = k.down;
  double w_part = use_rest ? weight[1] : weight[0], scan = wave_scan(w_part, lane), all = __shfl(scan, 63);
  if (use_rest && !(all > 0.0)) {
    use_rest = false;
    w_part = weight[0];
    scan = wave_scan(w_part, lane);
    all = __shfl(scan, 63);
  }
  const double at = (double)r * all;
  double before_part = __shfl_up(scan, 1);
  if (lane == 0) before_part = 0.0;
  const bool some = all > 0.0 && all <= 1.7976931348623157e308 && w_part > 0.0;
  const unsigned long long passed = __ballot(some && before_part + w_part > at), any = __ballot(some);
  const int part = passed ? __builtin_ctzll(passed) : any ? 63 - __builtin_clzll(any) : -1;
  const double left = at - __shfl(before_part, max(part, 0));
  if (part >= 0) {
    // the same inside the part, 2048 entries at a time
    const Rest<E> rest(a, b, n, k, sp, sq, s_table);
    const int hi = min(a.V, (part + 1) * a.part);
    double done = 0.0;
    int last = -1;
    Eight<E> vp, vq, next_p, next_q;
    const int first = part * a.part + 8 * threadIdx.x;
    if (first < hi) rest.fetch(first, a.V, use_rest, vp, vq);
    for (int i0 = part * a.part; i0 < hi; i0 += 8 * kThreads) {
      const int i = i0 + 8 * threadIdx.x;
      double p8[8], w[8], mine = 0.0;
      int hit = -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) p8[e] = w[e] = 0.0;
      if (i + 8 * kThreads < hi) rest.fetch(i + 8 * kThreads, a.V, use_rest, next_p, next_q);
      if (i < hi) rest.eight(i, use_rest, vp, vq, p8, w);
      if (!use_rest) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = p8[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        last = w[e] > 0.0 ? i + e : last;
        mine += w[e];
      }
      const double upto = wave_scan(mine, lane);
      if (lane == 63) s_wave[wid] = upto;
      __syncthreads();
      double before = done + (upto - mine);
      for (int v = 0; v < kWaves; ++v) {
        before += v < wid ? s_wave[v] : 0.0;
        done += s_wave[v];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        before += w[e];
        hit = hit < 0 && w[e] > 0.0 && before > left ? i + e : hit;
      }
      // the first lane's (a wave's lanes hold neighbouring entries), then the first wave's
      const unsigned long long hits = __ballot(hit >= 0);
      if (hits && lane == __builtin_ctzll(hits)) atomicMin(&s_token, hit);
      __syncthreads();
      if (s_token != INT_MAX) break;
      __syncthreads();
      vp = next_p;
      vq = next_q;
    }
    if (s_token == INT_MAX) {   // by rounding alone
#pragma unroll
      for (int j = 32; j >= 1; j >>= 1) last = max(last, __shfl_xor(last, j));
      if (lane == 0) atomicMax(&s_last, last);
      __syncthreads();
    }
  }
  const int token = part < 0 ? -1 : s_token == INT_MAX ? s_last : s_token;
  for (int t = threadIdx.x; t <= a.T; t += kThreads)
    a.out_token[(long long)b * (a.T + 1) + t] = t < n ? a.token[(long long)b * a.T + t] : t == n ? token : -1;
}

// One workgroup a sequence, a wave a row in turn, as in decide.
__global__ __launch_bounds__(kDecideWaves * 64) void k_verify_greedy(VerifyCall a) {
  const int b = blockIdx.x, lane = threadIdx.x & 63, wid = threadIdx.x >> 6, len = draft_len(a, b);
  __shared__ int s_n, s_best;
  if (threadIdx.x == 0) s_n = len;
  __syncthreads();
  int mine = INT_MAX, best = -1;
  for (int t = wid; t <= len; t += kDecideWaves) {
    RowPart v{0.0, -INFINITY, INT_MAX};
    if (lane < a.splits) v = a.stats[((long long)b * (a.T + 1) + t) * a.splits + lane];
    float m = v.m;
    int idx = v.idx;
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) {
      const float om = __shfl_xor(m, k);
      const int oi = __shfl_xor(idx, k);
      idx = om > m ? oi : om < m ? idx : min(idx, oi);
      m = fmaxf(m, om);
    }
    if (idx == INT_MAX) idx = -1;   // a row of -inf and NaN has no largest entry
    const bool same = t < len && idx >= 0 && a.token[(long long)b * a.T + t] == idx;
    if (lane == 0 && t < len) a.accept[(long long)b * a.T + t] = same ? 1.f : 0.f;
    if (mine == INT_MAX && !same) {
      mine = t;
      best = idx;
      if (lane == 0) atomicMin(&s_n, t);
    }
  }
  __syncthreads();
  const int n = s_n;
  if (lane == 0 && mine == n) {
    s_best = best;
    a.n_accept[b] = n;
  }
  __syncthreads();
  for (int t = len + threadIdx.x; t < a.T; t += kDecideWaves * 64) a.accept[(long long)b * a.T + t] = 0.f;
  for (int t = threadIdx.x; t <= a.T; t += kDecideWaves * 64)
    a.out_token[(long long)b * (a.T + 1) + t] = t < n ? a.token[(long long)b * a.T + t] : t == n ? s_best : -1;
}

template <class E>
hipError_t verify(const VerifyCall& a, hipStream_t s) {
  hipError_t e;
  const long long rows = (long long)a.B * (a.T + 1) + (a.draft && !a.greedy ? (long long)a.B * a.T : 0);
  if (a.greedy) {
    k_verify_stats<E, kGreedy><<<(unsigned)(rows * a.splits), kThreads, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    k_verify_greedy<<<a.B, kDecideWaves * 64, 0, s>>>(a);
    return hipGetLastError();
  }
  if (a.totals)
    k_verify_stats<E, kSingle><<<(unsigned)(rows * a.splits), kThreads, 0, s>>>(a);
  else
    k_verify_stats<E, kDouble><<<(unsigned)(rows * a.splits), kThreads, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (!a.totals) {
    k_verify_parts<E, true><<<(unsigned)(a.B * a.parts), kDecideWaves * 64, 0, s>>>(a);
  } else {
    k_verify_decide<E><<<a.B, kDecideWaves * 64, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    k_verify_totals<E><<<(unsigned)(a.B * a.parts), kThreads, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    k_verify_parts<E, false><<<(unsigned)(a.B * a.parts), kThreads, 0, s>>>(a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_verify_token<E><<<a.B, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyCall& a, hipStream_t s) {
  switch (a.dtype) {
    case RPD_DTYPE_BF16: return verify<Bf16>(a, s);
    case RPD_DTYPE_F16: return verify<F16>(a, s);
    default: return verify<F32>(a, s);
  }
}

}  // namespace rpd
