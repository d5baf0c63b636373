// Verification of drafted tokens against a target's logits, from given random
// numbers.
//
//   p_t = softmax(target_scale z_t), q_t = softmax(draft_scale y_t)
//   a_t = min(1, p_t(x_t) / q_t(x_t)); token t is accepted while u_t < a_t
//   after n accepted: w = max(0, p_n - q_n) if token n was turned down (p_n
//   where that is empty), p_n if the draft ended; the next token is the lowest
//   v with w_0 + .. + w_v > r sum w
//
// Bound: one read of the rows. The steps:
//   k_verify_stats   maximum and sum of a part of a row, every row at once
//                    (float32: an acceptance is off by about 1e-7)
//   k_verify_pick    each workgroup merges its sequence's statistics, finds n,
//                    and sums its part of row n in float64
//   k_verify_rest    the parts of sum w, float64 (only with draft logits)
//   k_verify_token   the part that r falls in, then the token in it
// The token's border lies among up to V cumulative sums a few 1e-6 apart, so
// these are float64 throughout, exponentials included: in float32 a draw in a
// hundred of a flat row would fall on the neighbour of the right token.
#include <cstdint>

#include "logit_rows.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr int kThreads = 256;

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
template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_stats(VerifyCall a) {
  const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits;
  const bool is_draft = row >= a.B * (a.T + 1);
  const int rr = is_draft ? row - a.B * (a.T + 1) : row, per = is_draft ? a.T : a.T + 1;
  const int b = rr / per, t = rr - b * per;
  if (is_draft ? t >= draft_len(a, b) : t > draft_len(a, b)) return;   // rows behind the draft are not read
  const typename E::t* p = is_draft ? draft_row<E>(a, b, t) : target_row<E>(a, b, t);
  const float scale = is_draft ? a.draft_scale : a.target_scale;
  const int lo = split * a.chunk, hi = min(a.V, lo + a.chunk);
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  __shared__ float2 s_part[kThreads / 64];
  if (a.greedy) {
    float m = -INFINITY;
    int idx = INT_MAX;
    for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
      const float z = E::one(p + i);
      const bool up = z > m;
      m = up ? z : m;
      idx = up ? i : idx;
    }
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) {
      const float om = __shfl_xor(m, k);
      const int oi = __shfl_xor(idx, k);
      idx = om > m ? oi : om < m ? idx : min(idx, oi);
      m = fmaxf(m, om);
    }
    if (lane == 0) s_part[wid] = make_float2(m, __int_as_float(idx));
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kThreads / 64; ++w) {
        const float om = s_part[w].x;
        const int oi = __float_as_int(s_part[w].y);
        idx = om > m ? oi : om < m ? idx : min(idx, oi);
        m = fmaxf(m, om);
      }
      a.stats[(long long)row * a.splits + split] = make_float2(m, __int_as_float(idx));
    }
    return;
  }
  MaxSum s{-INFINITY, 0.f};
  for (int i = lo + 8 * threadIdx.x; i < hi; i += 8 * kThreads) {
    float z[8];
    if (i + 8 <= hi) {
      Eight<E> v;
      v.load(p + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = v.at(e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = i + e < hi ? E::one(p + i + e) : -INFINITY;
    }
    maxsum_push(s, z, scale);
  }
  s = wave_maxsum(s, scale);
  if (lane == 0) s_part[wid] = make_float2(s.m, s.S);
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) s = maxsum_merge(s, MaxSum{s_part[w].x, s_part[w].y}, scale);
    a.stats[(long long)row * a.splits + split] = make_float2(s.m, s.S);
  }
}

// a row's statistics, merged by one wave in a fixed order
__device__ __forceinline__ MaxSum row_stats(const VerifyCall& a, long long row, float scale, int lane) {
  MaxSum s{-INFINITY, 0.f};
  for (int i = lane; i < a.splits; i += 64) {
    const float2 v = a.stats[row * a.splits + i];
    s = maxsum_merge(s, MaxSum{v.x, v.y}, scale);
  }
  return wave_maxsum(s, scale);
}

struct Pick {
  int n;           // accepted tokens
  int len;
  float mp, mq;    // references (scaled maxima) of the target's row n and, if turned down, the draft's
};

// what the sequence b comes to (the whole workgroup; s_acc: T + 1 floats of LDS, s_pick: one Pick)
template <class E>
__device__ __forceinline__ void decide(const VerifyCall& a, int b, bool write, Pick* s_pick) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int len = draft_len(a, b);
  __shared__ int s_first;
  if (threadIdx.x == 0) s_first = len;
  __syncthreads();
  for (int t = wid; t < len; t += kThreads / 64) {
    const MaxSum p = row_stats(a, (long long)b * (a.T + 1) + t, a.target_scale, lane);
    const int x = a.token[(long long)b * a.T + t];
    double l = -INFINITY;
    if (x >= 0 && x < a.V) {
      l = (double)E::one(target_row<E>(a, b, t) + x) * (double)a.target_scale - ref_of(p.m, a.target_scale) - log((double)p.S);
      if (a.draft) {
        const MaxSum q = row_stats(a, (long long)a.B * (a.T + 1) + (long long)b * a.T + t, a.draft_scale, lane);
        l -= (double)E::one(draft_row<E>(a, b, t) + x) * (double)a.draft_scale - ref_of(q.m, a.draft_scale) - log((double)q.S);
      }
    }
    const float acc = l > 0.0 ? 1.f : (float)exp(l);
    if (lane == 0) {
      if (write) a.accept[(long long)b * a.T + t] = acc;
      if (!(a.u[(long long)b * a.T + t] < acc)) atomicMin(&s_first, t);
    }
  }
  if (write)
    for (int t = len + threadIdx.x; t < a.T; t += kThreads) a.accept[(long long)b * a.T + t] = 0.f;
  __syncthreads();
  if (wid == 0) {
    const int n = s_first;
    const MaxSum p = row_stats(a, (long long)b * (a.T + 1) + n, a.target_scale, lane);
    MaxSum q{0.f, 0.f};
    if (a.draft && n < len) q = row_stats(a, (long long)a.B * (a.T + 1) + (long long)b * a.T + n, a.draft_scale, lane);
    if (lane == 0) *s_pick = Pick{n, len, ref_of(p.m, a.target_scale), ref_of(q.m, a.draft_scale)};
  }
  __syncthreads();
}

template <int N>
__device__ __forceinline__ void block_sum(double (&v)[N], double (*s)[N]) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) v[i] += __shfl_xor(v[i], k);
    if (lane == 0) s[wid][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) v[i] += s[w][i];
  }
}

// e^(scale z - m) of element v of a row
template <class E>
__device__ __forceinline__ double mass(const typename E::t* row, int v, float scale, float m) {
  return exp((double)E::one(row + v) * (double)scale - (double)m);
}

template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_pick(VerifyCall a) {
  const int part = blockIdx.x % a.parts, b = blockIdx.x / a.parts;
  __shared__ Pick s_pick;
  __shared__ double s_sum[kThreads / 64][3];
  decide<E>(a, b, part == 0, &s_pick);
  const Pick k = s_pick;
  const bool down = k.n < k.len;
  if (part == 0) {
    if (threadIdx.x == 0) a.n_accept[b] = k.n;
  }
  const int x = down ? a.token[(long long)b * a.T + k.n] : -1;
  const typename E::t* p = target_row<E>(a, b, k.n);
  const typename E::t* q = a.draft && down ? draft_row<E>(a, b, k.n) : nullptr;
  double v[3] = {0.0, 0.0, 0.0};   // target, draft, target without the drafted token
  const int hi = min(a.V, (part + 1) * a.part);
  for (int i = part * a.part + threadIdx.x; i < hi; i += kThreads) {
    const double e = mass<E>(p, i, a.target_scale, k.mp);
    v[0] += e;
    if (q) v[1] += mass<E>(q, i, a.draft_scale, k.mq);
    v[2] += i == x ? 0.0 : e;
  }
  block_sum(v, s_sum);
  if (threadIdx.x < 3) a.sums[((long long)threadIdx.x * a.B + b) * a.parts + part] = v[threadIdx.x];
}

// the total over the parts, in a fixed order
__device__ __forceinline__ double total(const VerifyCall& a, int which, int b) {
  double t = 0.0;
  for (int i = 0; i < a.parts; ++i) t += a.sums[((long long)which * a.B + b) * a.parts + i];
  return t;
}

struct Row {
  float mp, mq;
  double sp, sq;
};
// maxima and float64 sums of the rows that sequence b samples from
template <class E>
__device__ __forceinline__ Row sampled_row(const VerifyCall& a, int b, int n, bool down) {
  const int lane = threadIdx.x & 63;
  Row r;
  r.mp = ref_of(row_stats(a, (long long)b * (a.T + 1) + n, a.target_scale, lane).m, a.target_scale);
  r.mq = a.draft && down
             ? ref_of(row_stats(a, (long long)a.B * (a.T + 1) + (long long)b * a.T + n, a.draft_scale, lane).m, a.draft_scale)
             : 0.f;
  r.sp = total(a, 0, b);
  r.sq = total(a, 1, b);
  return r;
}

template <class E>
__device__ __forceinline__ double rest(const VerifyCall& a, const typename E::t* p, const typename E::t* q, int v,
                                       const Row& r) {
  const double w = mass<E>(p, v, a.target_scale, r.mp) / r.sp - mass<E>(q, v, a.draft_scale, r.mq) / r.sq;
  return w > 0.0 ? w : 0.0;
}

// the parts of sum max(0, p - q), over the sums of the target without the drafted token
template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_rest(VerifyCall a) {
  const int part = blockIdx.x % a.parts, b = blockIdx.x / a.parts;
  const int n = a.n_accept[b];
  if (n >= draft_len(a, b)) return;
  __shared__ double s_sum[kThreads / 64][1];
  const Row r = sampled_row<E>(a, b, n, true);
  const typename E::t *p = target_row<E>(a, b, n), *q = draft_row<E>(a, b, n);
  double v[1] = {0.0};
  const int hi = min(a.V, (part + 1) * a.part);
  for (int i = part * a.part + threadIdx.x; i < hi; i += kThreads) v[0] += rest<E>(a, p, q, i, r);
  block_sum(v, s_sum);
  if (threadIdx.x == 0) a.sums[(2LL * a.B + b) * a.parts + part] = v[0];
}

template <class E>
__global__ __launch_bounds__(kThreads) void k_verify_token(VerifyCall a) {
  const int b = blockIdx.x, n = a.n_accept[b];
  const bool down = n < draft_len(a, b);
  const int x = down ? a.token[(long long)b * a.T + n] : -1;
  __shared__ double s_scan[kThreads];
  __shared__ int s_part, s_token, s_last;
  __shared__ double s_left;
  const Row r = sampled_row<E>(a, b, n, down);
  const double sw = down ? total(a, 2, b) : 0.0;
  const bool use_rest = down && sw > 0.0;
  const double all = use_rest ? sw : r.sp;
  const double* parts = a.sums + ((use_rest ? 2LL : 0LL) * a.B + b) * a.parts;
  if (threadIdx.x == 0) {
    // the part in which the running sum passes r of the whole; by rounding alone, the last one that holds anything
    const double at = (double)a.r[b] * all;
    double before = 0.0;
    int pick = -1;
    s_left = 0.0;
    if (all > 0.0 && all <= 1.7976931348623157e308)
      for (int i = 0; i < a.parts; ++i) {
        if (parts[i] > 0.0) {
          pick = i;
          s_left = at - before;
          if (before + parts[i] > at) break;
        }
        before += parts[i];
      }
    s_part = pick;
    s_token = INT_MAX;
    s_last = -1;
  }
  __syncthreads();
  const int part = s_part;
  if (part >= 0) {
    const typename E::t* p = target_row<E>(a, b, n);
    const typename E::t* q = a.draft && down ? draft_row<E>(a, b, n) : nullptr;
    auto weight = [&](int v) -> double {
      if (!use_rest) return mass<E>(p, v, a.target_scale, r.mp);
      if (q) return rest<E>(a, p, q, v, r);
      return v == x ? 0.0 : mass<E>(p, v, a.target_scale, r.mp);
    };
    const int each = a.part / kThreads, lo = part * a.part + threadIdx.x * each, hi = min(a.V, lo + each);
    double mine = 0.0;
    int last = -1;
    for (int v = lo; v < hi; ++v) {
      const double w = weight(v);
      mine += w;
      last = w > 0.0 ? v : last;
    }
    s_scan[threadIdx.x] = mine;
    if (last >= 0) atomicMax(&s_last, last);
    __syncthreads();
    double before = 0.0;
    for (int i = 0; i < (int)threadIdx.x; ++i) before += s_scan[i];
    if (before + mine > s_left) {
      double run = before;
      for (int v = lo; v < hi; ++v) {
        const double w = weight(v);
        run += w;
        if (w > 0.0 && run > s_left) {
          atomicMin(&s_token, v);
          break;
        }
      }
    }
    __syncthreads();
  }
  const int token = part < 0 ? -1 : s_token == INT_MAX ? s_last : s_token;
  for (int t = threadIdx.x; t <= a.T; t += kThreads)
    a.out_token[(long long)b * (a.T + 1) + t] = t < n ? a.token[(long long)b * a.T + t] : t == n ? token : -1;
}

__global__ __launch_bounds__(64) void k_verify_greedy(VerifyCall a) {
  const int b = blockIdx.x, lane = threadIdx.x, len = draft_len(a, b);
  int n = 0, best = -1;
  bool running = true;
  for (int t = 0; t <= len; ++t) {
    float m = -INFINITY;
    int idx = INT_MAX;
    for (int i = lane; i < a.splits; i += 64) {
      const float2 v = a.stats[((long long)b * (a.T + 1) + t) * a.splits + i];
      const int oi = __float_as_int(v.y);
      idx = v.x > m ? oi : v.x < m ? idx : min(idx, oi);
      m = fmaxf(m, v.x);
    }
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
    if (running) {
      best = idx;
      n = t;
      running = same;
    }
  }
  if (lane == 0) a.n_accept[b] = n;
  for (int t = len + lane; t < a.T; t += 64) a.accept[(long long)b * a.T + t] = 0.f;
  for (int t = lane; t <= a.T; t += 64)
    a.out_token[(long long)b * (a.T + 1) + t] = t < n ? a.token[(long long)b * a.T + t] : t == n ? best : -1;
}

template <class E>
hipError_t verify(const VerifyCall& a, hipStream_t s) {
  hipError_t e;
  const long long rows = (long long)a.B * (a.T + 1) + (a.draft && !a.greedy ? (long long)a.B * a.T : 0);
  k_verify_stats<E><<<(unsigned)(rows * a.splits), kThreads, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.greedy) {
    k_verify_greedy<<<a.B, 64, 0, s>>>(a);
    return hipGetLastError();
  }
  k_verify_pick<E><<<(unsigned)(a.B * a.parts), kThreads, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.draft && a.T > 0) {
    k_verify_rest<E><<<(unsigned)(a.B * a.parts), kThreads, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
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
