// Distillation from a teacher's top logits: loss and gradient of a row z of
// the student's logits, q = softmax(scale z).
//
//   p_j over the list of the teacher's tokens i_j: softmax of scale t_j over
//   the list, or with the teacher's log-sum-exp e^(scale t_j - lse), the rest
//   p_T = 1 - sum p_j being one entry for the tokens outside the list (mass
//   q_T of the student)
//   loss = sum_j p_j (ln p_j - ln q_{i_j}) + p_T (ln p_T - ln q_T)
//   d loss / d z_v = scale [ P q_v - (sum of p_j with i_j = v) ]     in the list
//                    scale [ (P - p_T / q_T) q_v ]                  outside
//   with P = sum p_j + p_T
//
// Bound: one read of z for the loss, one read and one write for the gradient.
// The student's mass outside the list is summed by itself (a bit of LDS per
// vocabulary entry marks the list): what is left of 1 after the list's mass is
// taken off would be rounding where the student is sure. The teacher's few
// probabilities and the loss are float64.
#include <cstdint>

#include "logit_rows.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 4;   // vectors that a thread holds
constexpr int kMaxList = RPD_DISTILL_MAX_K;
static_assert(kMaxList <= kThreads, "a thread an entry of the list");

// a row's state between the loss and the gradient
struct RowState {
  float top, in;   // in the list: in * e^(scale (z - top)) - p, with in = P / S (S relative to top)
  float tail, out; // outside: out * e^(scale (z - tail)), tail the largest logit there (a student that is
                   // sure leaves e^(scale (tail - top)) far below float32's range)
  float tref;      // the teacher's p_j = tinv * e^(scale (t_j - tref)), with its log-sum-exp e^(scale t_j - tref)
  float tinv;
  float any;       // 0: no gradient
};
static_assert(sizeof(RowState) <= RPD_DISTILL_STATE * sizeof(float), "the state that callers allocate");

__device__ __forceinline__ float teacher_at(const DistillCall& a, long long i) {
  if (a.teacher_dtype == RPD_DTYPE_F32) return static_cast<const float*>(a.teacher)[i];
  return a.teacher_dtype == RPD_DTYPE_BF16 ? Bf16::one(static_cast<const uint16_t*>(a.teacher) + i)
                                           : F16::one(static_cast<const uint16_t*>(a.teacher) + i);
}

// the exponent of a teacher's logit relative to tref
__device__ __forceinline__ double teacher_below(const DistillCall& a, double t, float tref) {
  return a.lse ? t * (double)a.scale - (double)tref : (t - (double)tref) * (double)a.scale;
}

__device__ __forceinline__ bool skipped(const DistillCall& a, int n) { return a.weight && a.weight[n] == 0.f; }

template <class E>
__device__ __forceinline__ const typename E::t* row_of(const DistillCall& a, int n) {
  return static_cast<const typename E::t*>(a.logits) + n * a.stride;
}

// A list in LDS is read four at a time: filled up with -1.
__device__ __forceinline__ int4 four_of(const int* s_ids, int i) { return *reinterpret_cast<const int4*>(s_ids + i); }

// the row's list into LDS; with `marks` (a bit per entry of [lo, hi)), those in it marked. Ends with a barrier.
__device__ __forceinline__ void load_list(const DistillCall& a, int n, int* s_ids, uint32_t* s_mark, int lo, int hi) {
  if (s_mark)
    for (int i = threadIdx.x; i < (hi - lo + 31) / 32; i += blockDim.x) s_mark[i] = 0;
  for (int j = threadIdx.x; j < (a.k + 3 & ~3); j += blockDim.x) s_ids[j] = j < a.k ? a.ids[(long long)n * a.k + j] : -1;
  __syncthreads();
  if (!s_mark) return;
  for (int j = threadIdx.x; j < a.k; j += blockDim.x) {
    const int v = s_ids[j];
    if (v >= lo && v < hi) atomicOr(&s_mark[(v - lo) >> 5], 1u << ((v - lo) & 31));
  }
  __syncthreads();
}

// maximum and mass of the entries of a part of a row outside the list
template <class E>
__global__ __launch_bounds__(kThreads) void k_distill_part(DistillCall a) {
  const int n = blockIdx.x / a.splits, split = blockIdx.x - n * a.splits;
  if (skipped(a, n)) return;
  extern __shared__ uint32_t s_mark[];   // a bit per entry of the part
  __shared__ __align__(16) int s_ids[kMaxList];
  __shared__ float s_max[kThreads / 64], s_sum[kThreads / 64];
  const int lo = split * a.chunk, hi = min(a.V, lo + a.chunk);
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, first = lo + 8 * threadIdx.x;
  const typename E::t* p = row_of<E>(a, n);
  MaxSum s{-INFINITY, 0.f};
  Eight<E> held[kHeld];
  auto fetch = [&](int base) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (base + j * 8 * kThreads < hi) load_eight<E>(p, base + j * 8 * kThreads, hi, held[j]);
  };
  fetch(first);   // before the list, whose loads and barriers then cost nothing
  load_list(a, n, s_ids, s_mark, lo, hi);
  for (int base = first; base - 8 * (int)threadIdx.x < hi;) {
    // the list's entries out, then one maximum and one sum over all that are held
    float m = s.m;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = base + j * 8 * kThreads;
      if (i >= hi) continue;
      const uint32_t mark = s_mark[(i - lo) >> 5] >> ((i - lo) & 31) & 255u;
      if (mark) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = mark >> e & 1u ? -INFINITY : held[j].at(e);
        held[j].set(z);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, held[j].at(e));
    }
    const float top = top_of(m);
    s.S *= carry(s.m, top, a.scale);
    s.m = m;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      if (base + j * 8 * kThreads >= hi) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) s.S += exp_below(held[j].at(e), top, a.scale);
    }
    base += kHeld * 8 * kThreads;
    fetch(base);   // a part that is longer than a thread holds
  }
  float m = s.m;
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  if (lane == 0) s_max[wid] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, s_max[w]);
  float S = s.S * carry(s.m, top_of(m), a.scale);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) S += __shfl_xor(S, k);
  if (lane == 0) s_sum[wid] = S;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) S += s_sum[w];
    a.partials[(long long)n * a.splits + split] = make_float2(m, S);
  }
}

template <int N>
__device__ __forceinline__ void wave_sum(double (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) v[i] += __shfl_xor(v[i], k);
}

// The row's loss and state, by one wave: from the maximum and mass of its parts' entries outside the list. Latency is
// all of it: what needs no token is fetched at once, then the tokens' logits (1024 rows with a list of 64: 8.6 us, 12.5
// with five waits for memory instead of two).
template <class E>
__global__ __launch_bounds__(64) void k_distill_loss(DistillCall a) {
  constexpr int kEach = kMaxList / 64;
  const int n = blockIdx.x, lane = threadIdx.x;
  __shared__ __align__(16) int s_ids[kMaxList];
  float weight = a.weight ? a.weight[n] : 1.f;
  const float tref_given = a.lse ? a.lse[n] : 0.f;
  float2 part = make_float2(-INFINITY, 0.f);   // (at most 64 parts a row)
  if (lane < a.splits) part = a.partials[(long long)n * a.splits + lane];
  float teacher[kEach];
  int at[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int j = lane + 64 * u;
    at[u] = -1;
    teacher[u] = 0.f;
    if (j < a.k) {
      at[u] = a.ids[(long long)n * a.k + j];
      teacher[u] = teacher_at(a, (long long)n * a.k + j);
    }
  }
  asm volatile("" : "+v"(weight), "+v"(part.x), "+v"(part.y), "+v"(at[0]), "+v"(teacher[0]));   // before the branch
  if (weight == 0.f) {
    if (lane == 0) {
      a.loss[n] = 0.f;
      *reinterpret_cast<RowState*>(a.state + (long long)n * RPD_DISTILL_STATE) = RowState{};
    }
    return;
  }
  const typename E::t* p = row_of<E>(a, n);
  double t[kEach], z[kEach], pj[kEach];
  bool ok[kEach], first[kEach];
  MaxSum s{part.x, 0.f};
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) s.m = fmaxf(s.m, __shfl_xor(s.m, k));
  s.S = part.y * carry(part.x, top_of(s.m), a.scale);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) s.S += __shfl_xor(s.S, k);
  double sums[2] = {0.0, 0.0};   // teacher's, student's mass in the list
  float tmax = -INFINITY, zmax = s.m;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int v = at[u];
    s_ids[lane + 64 * u] = v;
    ok[u] = v >= 0 && v < a.V;
    const float tj = ok[u] ? teacher[u] : -INFINITY, zj = ok[u] ? E::one(p + v) : -INFINITY;
    t[u] = tj;
    z[u] = zj;
    tmax = fmaxf(tmax, tj);
    zmax = fmaxf(zmax, zj);
    first[u] = ok[u];
  }
  __syncthreads();
  // a token listed twice is in the list once
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int j = lane + 64 * u;
    if (64 * u >= a.k) continue;
#pragma unroll 4
    for (int i = 0; i < min(a.k, 64 * u + 64); i += 4) {
      const int4 v = four_of(s_ids, i);
      first[u] &= !((v.x == at[u] && i < j) || (v.y == at[u] && i + 1 < j) || (v.z == at[u] && i + 2 < j) ||
                    (v.w == at[u] && i + 3 < j));
    }
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) zmax = fmaxf(zmax, __shfl_xor(zmax, k));
  const float top = top_of(zmax), tail = top_of(s.m);
  const double scale = a.scale;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    if (64 * u >= a.k) continue;
    z[u] = (z[u] - (double)top) * scale;
    if (first[u]) sums[1] += exp(z[u]);
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) tmax = fmaxf(tmax, __shfl_xor(tmax, k));
  const float tref = a.lse ? tref_given : top_of(tmax);
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    pj[u] = 0.0;
    if (64 * u >= a.k) continue;
    t[u] = teacher_below(a, t[u], tref);
    if (ok[u]) pj[u] = exp(t[u]);
    sums[0] += pj[u];
  }
  wave_sum(sums);
  int listed = 0;   // different tokens in the list
#pragma unroll
  for (int u = 0; u < kEach; ++u)
    if (64 * u < a.k) listed += __popcll(__ballot(first[u]));
  // a list without any mass: in list mode there is no teacher, and no loss
  const bool none = !a.lse && sums[0] == 0.0;
  const double tinv = a.lse ? 1.0 : none ? 0.0 : 1.0 / sums[0];
  // NaN in the list shows in its own terms; where no token is outside the list, 1 - sum p is the rounding of lse
  const double rest = a.lse && listed < a.V ? fmax(0.0, 1.0 - sums[0]) : 0.0;
  const double drop = s.S == 0.f ? 0.0 : ((double)tail - (double)top) * scale;   // S_T's exponent in units of S's
  const double e_drop = exp(drop), S = (double)s.S * e_drop + sums[1];
  // four logarithms for the time of one
  const double logs = log(lane == 0 ? S : lane == 1 ? tinv : lane == 2 ? rest : (double)s.S);
  const double ln_S = __shfl(logs, 0), ln_tinv = __shfl(logs, 1), ln_rest = __shfl(logs, 2), ln_tail = __shfl(logs, 3);
  double l[1] = {0.0};
#pragma unroll
  for (int u = 0; u < kEach; ++u)
    if (pj[u] != 0.0) l[0] += pj[u] * tinv * ((t[u] + ln_tinv) - (z[u] - ln_S));
  wave_sum(l);
  if (lane != 0) return;
  if (rest > 0.0) l[0] += rest * (ln_rest - (ln_tail + drop - ln_S));
  const double P = (none ? 0.0 : sums[0] * tinv) + rest;
  a.loss[n] = none ? 0.f : (float)((double)weight * l[0]);
  RowState st;
  st.top = top;
  st.in = (float)(P / S);
  st.tail = tail;
  st.out = (float)(P * e_drop / S - (rest > 0.0 ? rest / (double)s.S : 0.0));
  st.tref = tref;
  st.tinv = (float)tinv;
  st.any = none ? 0.f : 1.f;
  *reinterpret_cast<RowState*>(a.state + (long long)n * RPD_DISTILL_STATE) = st;
}

// The part [lo, hi) of a row's gradient: the formula of the entries outside the list everywhere, then those in the
// list over it. Streamed past the caches, which keep the logits between the loss and the gradient. 1024 rows of 126464
// bf16, three quarters of them read: 40 us for the sums and 69 here (452 MB: 6.5 TB/s); with ordinary stores the sums
// take 14 us more, this 2.
template <class E>
__device__ __forceinline__ void row_grad(const DistillCall& a, int n, int lo, int hi, const RowState& st) {
  typedef typename E::t T;
  const T* p = row_of<E>(a, n);
  T* g = static_cast<T*>(a.grad) + n * a.grad_stride;
  const float c = (a.weight ? a.weight[n] : 1.f) * (a.up ? a.up[n] : 1.f) * a.scale, co = c * st.out;
  const int first = lo + 8 * threadIdx.x;
  Eight<E> held[kHeld];
  auto fetch = [&](int base) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (base + j * 8 * kThreads < hi) load_eight<E>(p, base + j * 8 * kThreads, hi, held[j]);
  };
  fetch(first);
  // a thread's entry of the list (kMaxList is no more than the threads), and its logits
  __shared__ __align__(16) int s_ids[kMaxList];
  load_list(a, n, s_ids, nullptr, 0, 0);
  const int mine = threadIdx.x, v = mine < a.k ? s_ids[mine] : -1;
  const bool here = v >= lo && v < hi;
  float zv = 0.f, tv = 0.f;
  if (here) {
    zv = E::one(p + v);
    tv = teacher_at(a, (long long)n * a.k + mine);
  }
  for (int base = first; base < hi;) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = base + j * 8 * kThreads;
      if (i >= hi) continue;
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = co * exp_below(held[j].at(e), st.tail, a.scale);
      if (i + 8 <= hi) {
        held[j].set(d);
        held[j].stream(g + i);
      } else {
        for (int e = 0; e < hi - i; ++e) g[i + e] = E::to(d[e]);
      }
    }
    base += kHeld * 8 * kThreads;
    fetch(base);
  }
  __syncthreads();
  if (!here) return;
  // the teacher's probability, of a token listed twice their sum, written once
  double pv = 0.0;
  bool first_of = true;
#pragma unroll 4
  for (int i = 0; i < a.k; i += 4) {
    const int4 q = four_of(s_ids, i);
    if (q.x != v && q.y != v && q.z != v && q.w != v) continue;
    for (int e = i; e < i + 4; ++e)
      if (s_ids[e] == v) {
        first_of &= e >= mine;
        const float t = e == mine ? tv : teacher_at(a, (long long)n * a.k + e);
        pv += exp(teacher_below(a, t, st.tref));
      }
  }
  if (first_of) g[v] = E::to(c * (st.in * exp_below(zv, st.top, a.scale) - (float)(pv * (double)st.tinv)));
}
template <class E>
__device__ __forceinline__ void row_zero(const DistillCall& a, int n, int lo, int hi) {
  typedef typename E::t T;
  T* g = static_cast<T*>(a.grad) + n * a.grad_stride;
  const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  Eight<E> v;
  v.set(none);
  for (int i = lo + 8 * threadIdx.x; i < hi; i += 8 * kThreads) {
    if (i + 8 <= hi)
      v.stream(g + i);
    else
      for (int e = i; e < hi; ++e) g[e] = E::to(0.f);
  }
}

template <class E>
__global__ __launch_bounds__(kThreads) void k_distill_grad(DistillCall a) {
  const int n = blockIdx.x / a.splits, split = blockIdx.x - n * a.splits;
  const int lo = split * a.chunk, hi = min(a.V, lo + a.chunk);
  const RowState st = *reinterpret_cast<const RowState*>(a.state + (long long)n * RPD_DISTILL_STATE);
  if (skipped(a, n) || st.any == 0.f) return row_zero<E>(a, n, lo, hi);   // such a row is not read
  row_grad<E>(a, n, lo, hi, st);
}

template <class E>
hipError_t loss_t(const DistillCall& a, hipStream_t s) {
  hipError_t e;
  k_distill_part<E><<<(unsigned)((long long)a.N * a.splits), kThreads, (size_t)(a.chunk + 31) / 32 * 4, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_distill_loss<E><<<a.N, 64, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || !a.grad) return e;
  k_distill_grad<E><<<(unsigned)((long long)a.N * a.splits), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class E>
hipError_t grad_t(const DistillCall& a, hipStream_t s) {
  k_distill_grad<E><<<(unsigned)((long long)a.N * a.splits), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_distill_loss(const DistillCall& a, hipStream_t s) {
  switch (a.dtype) {
    case RPD_DTYPE_BF16: return loss_t<Bf16>(a, s);
    case RPD_DTYPE_F16: return loss_t<F16>(a, s);
    default: return loss_t<F32>(a, s);
  }
}

hipError_t launch_distill_grad(const DistillCall& a, hipStream_t s) {
  switch (a.dtype) {
    case RPD_DTYPE_BF16: return grad_t<Bf16>(a, s);
    case RPD_DTYPE_F16: return grad_t<F16>(a, s);
    default: return grad_t<F32>(a, s);
  }
}

}  // namespace rpd
