// C ABI of sampling: argument validation. Kernels live in sample.hip.
#include "rpd_checks.h"

using namespace rpd;

namespace {

bool shape_ok(const rpd_sample* p) { return p->N >= 0 && p->N < 1 << 22 && p->V >= 1 && p->V <= 1 << 20; }

}  // namespace

extern "C" {

// a row is one workgroup's work, in its registers and LDS
size_t rpd_sample_workspace_size(const rpd_sample*) { return 0; }

rpd_status rpd_sample_tokens(const rpd_sample* p, void* /*workspace*/, size_t /*workspace_bytes*/, void* stream) {
  clear_error();
  if (!p) return fail(RPD_ERR_NULL_POINTER, "problem is NULL");
  if (!shape_ok(p)) return fail(RPD_ERR_BAD_SHAPE, "need 0<=N<2^22, 1<=V<=2^20 (got N=%d V=%d)", p->N, p->V);
  if (!is_float_dtype(p->dtype)) return fail(RPD_ERR_UNSUPPORTED, "dtype %d is not supported", p->dtype);
  if (!p->scales && !(p->logit_scale >= 0.f && p->logit_scale <= kSampleMaxScale))
    return fail(RPD_ERR_BAD_PARAM, "logit_scale must be > 0 and at most 2^100, or 0 for 1 (got %g)", p->logit_scale);
  if (!p->top_ks && p->top_k < 0) return fail(RPD_ERR_BAD_PARAM, "top_k must be >= 0 (got %d)", p->top_k);
  if (!p->top_ps && !(p->top_p > 0.f)) return fail(RPD_ERR_BAD_PARAM, "top_p must be > 0 (got %g)", p->top_p);
  if (!p->min_ps && !(p->min_p >= 0.f && p->min_p <= 1.f))
    return fail(RPD_ERR_BAD_PARAM, "min_p must be in 0..1 (got %g)", p->min_p);
  if (p->logits_stride < p->V || (p->filtered && p->filtered_stride < p->V))
    return fail(RPD_ERR_BAD_SHAPE, "row strides must be at least V");
  if (p->N == 0) return RPD_OK;
  if (!p->logits || !p->r || !p->token) return fail(RPD_ERR_NULL_POINTER, "logits, r and token are required");
  const unsigned e = elem_align(p->dtype);
  if (misaligned(p->logits, e) || misaligned(p->filtered, e) || misaligned(p->r, 3) || misaligned(p->scales, 3) ||
      misaligned(p->top_ks, 3) || misaligned(p->top_ps, 3) || misaligned(p->min_ps, 3) || misaligned(p->token, 3) ||
      misaligned(p->prob, 3) || misaligned(p->kept, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  const int size = size_of(p->dtype);
  if (p->filtered && rows_meet(p->logits, p->logits_stride * size, (long long)p->V * size, p->filtered,
                               p->filtered_stride * size, (long long)p->V * size, p->N))
    return fail(RPD_ERR_BAD_PARAM, "filtered must not overlap the logits");
  SampleCall a{};
  a.N = p->N;
  a.V = p->V;
  a.dtype = p->dtype;
  a.logits = p->logits;
  a.stride = p->logits_stride;
  a.r = p->r;
  a.scale = scale_of(p->logit_scale);
  a.top_k = p->top_k;
  a.top_p = p->top_p;
  a.min_p = p->min_p;
  a.scales = p->scales;
  a.top_ks = p->top_ks;
  a.top_ps = p->top_ps;
  a.min_ps = p->min_ps;
  a.token = p->token;
  a.prob = p->prob;
  a.kept = p->kept;
  a.filtered = p->filtered;
  a.filtered_stride = p->filtered_stride;
  const hipError_t st = launch_sample(a, static_cast<hipStream_t>(stream));
  if (st != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(st));
  return RPD_OK;
}

}  // extern "C"
