// C ABI of the operators around the commit step: argument validation,
// workspace layout and launch planning. Kernels live in quant.hip, verify.hip
// and distill.hip.
#include <algorithm>
#include <cmath>

#include "rpd_checks.h"

using namespace rpd;

namespace {

// ------------------------------------------------------------------ quant --

bool quant_shape_ok(const rpd_quant_head* h) {
  return h->V >= 1 && h->V < (1 << 28) && h->d >= 8 && h->d <= (1 << 20) && h->d % 8 == 0 &&
         (long long)h->V * h->d <= 1LL << 36;
}
bool quant_ok(const rpd_quant_head* h) {
  return quant_shape_ok(h) && (h->group == 32 || h->group == 64 || h->group == 128) &&
         (h->dtype == RPD_DTYPE_BF16 || h->dtype == RPD_DTYPE_F16) && (h->has_zeros == 0 || h->has_zeros == 1);
}

rpd::QuantDims quant_dims(const rpd_quant_head* h) {
  rpd::QuantDims q{};
  q.V = h->V;
  q.d = h->d;
  q.group = h->group;
  q.ng = (h->d + h->group - 1) / h->group;
  q.vt = (h->V + 15) / 16;
  q.nc = (h->d + 127) / 128;
  q.ngp = q.nc * (128 / h->group);
  const size_t entries = (size_t)q.vt * 16 * q.ngp;
  q.scale_offset = round256((size_t)q.vt * q.nc * 1024);
  q.zero_offset = q.scale_offset + round256(entries * 2);
  q.bytes = q.zero_offset + (h->has_zeros ? round256(entries) : 0);
  return q;
}

// Workgroups of up to 16 waves, each wave keeping the x of 1, 2 or 4 chunks of
// 128 columns in registers; longer rows take several rounds and reload x. Rows
// of V = 126464 bf16, us: 4096 columns with 16 waves 43.4 (1 row) and 51.0 (16
// rows), with 8 waves of twice the chunks 44.3 and 54.2 (2048 columns: 26.8 and
// 31.1, 25.9 and 30.0). More than 16 rows share converted codes between two
// tiles of 16 as long as their x fits the registers: 32 rows of 4096 columns
// 63.4, of 2048 41.0, and 77.1 and 49.4 as row groups of 16; 64 rows 102.8 and
// 132.7.
void quant_plan(const rpd::QuantDims& q, rpd::QuantCall& a) {
  a.nc_wave = q.nc <= 16 ? 1 : q.nc <= 32 ? 2 : 4;
  a.row_tiles = a.M > 16 && a.nc_wave < 4 ? 2 : 1;
  a.row_groups = (int)up_div(a.M, 16 * a.row_tiles);
  a.waves = std::min(16, (int)up_div(q.nc, a.nc_wave));
  a.rounds = (int)up_div(q.nc, a.waves * a.nc_wave);
  const int per_cu = std::max(1, 16 / a.waves);
  const int most = std::max(8, 256 * per_cu / a.row_groups / 8 * 8);
  a.slots = std::min(most, (int)up_div(q.vt, 8) * 8);
}

// Workspace of a call: the laid out rows (more than 16 of them), then the states of the statistics.
struct QuantSpace {
  size_t exps, states, bytes;   // offsets (the rows come first)
};
QuantSpace quant_space(const rpd::QuantDims& q, const rpd::QuantCall& a) {
  QuantSpace w{};
  if (a.M > 16) {
    const size_t tiles = (size_t)a.row_groups * a.row_tiles;
    w.exps = tiles * q.nc * 4096;
    w.states = w.exps + round256(tiles * 64);
  }
  w.bytes = w.states + (a.stats ? round256((size_t)a.M * a.slots * 16) : 0);
  return w;
}

rpd_status check_head(const rpd_quant_head* h) {
  if (!h) return fail(RPD_ERR_NULL_POINTER, "head is NULL");
  if (!quant_shape_ok(h))
    return fail(RPD_ERR_BAD_SHAPE, "need 1<=V<2^28, 8<=d<=2^20, d%%8==0, V*d<=2^36 (got V=%d d=%d)", h->V, h->d);
  if (h->dtype != RPD_DTYPE_BF16 && h->dtype != RPD_DTYPE_F16)
    return fail(RPD_ERR_UNSUPPORTED, "head dtype %d is not supported (bf16 or fp16)", h->dtype);
  if (h->group != 32 && h->group != 64 && h->group != 128)
    return fail(RPD_ERR_UNSUPPORTED, "group %d is not supported (32, 64 or 128)", h->group);
  if (h->has_zeros != 0 && h->has_zeros != 1) return fail(RPD_ERR_BAD_PARAM, "has_zeros must be 0 or 1");
  return RPD_OK;
}

// ----------------------------------------------------------------- verify --

bool verify_shape_ok(const rpd_verify* p) {
  return p->B >= 1 && p->T >= 0 && p->V >= 1 && p->V <= (1 << 28) && (long long)p->B * ((long long)p->T + 1) <= 1 << 20;
}

constexpr long long kFill = 4096;   // workgroups of 256 threads: 256 CUs, 8 on each, twice

// Logits from which float32 statistics, and a pass of float64 sums over the sampled rows, beat float64 statistics:
// 4 drafted tokens, V = 126464, bf16: 8 sequences (9.1 million logits) take 30.5 us so and 28.0 in float64, 16 take
// 36.4 and 41.0, 32 take 45.7 and 64.2.
constexpr long long kSingleStats = 12000000;

struct VerifyPlan {
  int splits, chunk, parts, part;
  long long rows;
  bool single;                         // statistics in float32
  size_t picks, sums, totals, bytes;   // workspace offsets
};

VerifyPlan verify_plan(const rpd_verify* p) {
  VerifyPlan v{};
  const bool greedy = (p->flags & RPD_VERIFY_GREEDY) != 0;
  v.rows = (long long)p->B * (p->T + 1) + (p->draft && !greedy ? (long long)p->B * p->T : 0);
  // Parts of whole 2048 entries (8 a thread), at most 64 of them, which one wave merges in a step. For the
  // statistics, as long as the launch fills the GPU's workgroups twice over, they are doubled while shorter than
  // 8192, which a workgroup's threads hold in registers: 288 target and 256 draft rows of 152064 bf16 63.0 us, with
  // parts of 4096 68.5; 1024 rows of 126464 bf16 distilled 137 us, with parts of 2048 191. From V = 262145 to 393216
  // parts of 6144 become 12288, read in two rounds (the verification's, twice): 1024 rows of 393216 bf16 distilled
  // 448 us and greedily verified 141, in parts of 6144 504 and 148; of 300001, 350 and 106, and 340 and 117.
  v.part = (int)up_div(up_div(p->V, 64), 2048) * 2048;
  v.chunk = v.part;
  while (p->B * up_div(p->V, v.part) > kMaxBlocks) v.part *= 2;   // so many sequences that a launch holds no more
  v.parts = (int)up_div(p->V, v.part);
  while (v.chunk < 8192 && v.rows * up_div(p->V, 2 * v.chunk) >= kFill) v.chunk *= 2;
  v.splits = (int)up_div(p->V, v.chunk);
  v.picks = round256((size_t)v.rows * v.splits * sizeof(rpd::RowPart));
  v.sums = v.picks + round256((size_t)p->B * sizeof(rpd::VerifyPick));
  const size_t sums = round256((size_t)2 * p->B * v.parts * sizeof(double));
  v.single = v.rows * p->V >= kSingleStats;
  v.totals = v.sums + sums;
  v.bytes = greedy ? v.picks : v.totals + (v.single ? sums : 0);
  return v;
}

// ---------------------------------------------------------------- distill --

bool distill_shape_ok(const rpd_distill* p) {
  return p->N >= 0 && p->N < 1 << 24 && p->V >= 1 && p->V <= 1 << 20 && p->k >= 1 && p->k <= RPD_DISTILL_MAX_K;
}

struct DistillPlan {
  int splits, chunk;
  size_t bytes;
};

DistillPlan distill_plan(const rpd_distill* p) {
  DistillPlan d{};
  // parts as the verification's statistics are cut
  d.chunk = (int)up_div(up_div(p->V, 64), 2048) * 2048;
  while (d.chunk < 8192 && p->N * up_div(p->V, 2 * d.chunk) >= kFill) d.chunk *= 2;
  d.splits = (int)up_div(p->V, d.chunk);
  d.bytes = round256((size_t)p->N * d.splits * 8);
  return d;
}

// Whether a row of the gradient takes memory of a row of the logits, which other workgroups still read then (both
// aligned to their elements). Rows of one stride may lie between each other; of two strides, the ranges must be apart.
bool grad_over_logits(const rpd_distill* p) {
  const long long size = p->dtype == RPD_DTYPE_F32 ? 4 : 2, V = p->V, last = p->N - 1;
  const __int128 at =
      ((__int128) reinterpret_cast<uintptr_t>(p->grad) - (__int128) reinterpret_cast<uintptr_t>(p->logits)) / size;
  if (at >= (__int128)last * p->logits_stride + V || -at >= (__int128)last * p->grad_stride + V) return false;
  if (last == 0 || p->grad_stride != p->logits_stride) return true;
  const long long stride = p->logits_stride, shift = (long long)(((at % stride) + stride) % stride);
  return shift < V || shift > stride - V;
}

rpd_status check_distill(const rpd_distill* p, bool grad) {
  if (!p) return fail(RPD_ERR_NULL_POINTER, "problem is NULL");
  if (!distill_shape_ok(p))
    return fail(RPD_ERR_BAD_SHAPE, "need 0<=N<2^24, 1<=V<=2^20, 1<=k<=%d (got N=%d V=%d k=%d)", RPD_DISTILL_MAX_K, p->N,
                p->V, p->k);
  if (!is_float_dtype(p->dtype) || !is_float_dtype(p->teacher_dtype))
    return fail(RPD_ERR_UNSUPPORTED, "dtype %d / teacher_dtype %d is not supported", p->dtype, p->teacher_dtype);
  if (!std::isfinite(p->logit_scale) || p->logit_scale < 0.f)
    return fail(RPD_ERR_BAD_PARAM, "logit_scale must be finite and > 0, or 0 for 1 (got %g)", p->logit_scale);
  if (p->logits_stride < p->V || (grad && p->grad_stride < p->V))
    return fail(RPD_ERR_BAD_SHAPE, "row strides must be at least V");
  if ((long long)p->N * distill_plan(p).splits > kMaxBlocks)
    return fail(RPD_ERR_BAD_SHAPE, "N * V is too large (N=%d V=%d)", p->N, p->V);
  if (p->N == 0) return RPD_OK;
  if (!p->logits || !p->id || !p->teacher || !p->state || (grad && !p->grad))
    return fail(RPD_ERR_NULL_POINTER, "logits, id, teacher, state%s are required", grad ? " and grad" : "");
  const unsigned e = elem_align(p->dtype);
  if (misaligned(p->logits, e) || misaligned(p->grad, e) || misaligned(p->teacher, elem_align(p->teacher_dtype)) ||
      misaligned(p->id, 3) || misaligned(p->teacher_lse, 3) || misaligned(p->weight, 3) ||
      misaligned(p->grad_loss, 3) || misaligned(p->loss, 3) || misaligned(p->state, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  if (grad && grad_over_logits(p)) return fail(RPD_ERR_BAD_PARAM, "grad must not be the logits' memory");
  return RPD_OK;
}

rpd::DistillCall distill_call(const rpd_distill* p, void* ws) {
  const DistillPlan d = distill_plan(p);
  rpd::DistillCall a{};
  a.N = p->N;
  a.V = p->V;
  a.k = p->k;
  a.dtype = p->dtype;
  a.teacher_dtype = p->teacher_dtype;
  a.logits = p->logits;
  a.stride = p->logits_stride;
  a.ids = p->id;
  a.teacher = p->teacher;
  a.lse = p->teacher_lse;
  a.weight = p->weight;
  a.up = p->grad_loss;
  a.scale = scale_of(p->logit_scale);
  a.loss = p->loss;
  a.state = p->state;
  a.grad = p->grad;
  a.grad_stride = p->grad_stride;
  a.partials = static_cast<float2*>(ws);
  a.splits = d.splits;
  a.chunk = d.chunk;
  return a;
}

}  // namespace

extern "C" {

size_t rpd_quant_packed_size(const rpd_quant_head* h) {
  if (!h || !quant_ok(h)) return 0;
  return quant_dims(h).bytes;
}

rpd_status rpd_quant_pack(const rpd_quant_head* h, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                          void* packed, size_t packed_bytes, void* stream) {
  rpd::clear_error();
  rpd_status st = check_head(h);
  if (st != RPD_OK) return st;
  if (!codes || !scales || !packed) return fail(RPD_ERR_NULL_POINTER, "codes, scales and packed are required");
  if (h->has_zeros ? !zeros : zeros != nullptr)
    return fail(RPD_ERR_NULL_POINTER, "zeros must be given exactly with has_zeros");
  if (misaligned(scales, 1)) return fail(RPD_ERR_UNSUPPORTED, "scales must be aligned to their element");
  const rpd::QuantDims q = quant_dims(h);
  if (misaligned(packed, 255)) return fail(RPD_ERR_UNSUPPORTED, "packed must be 256-byte aligned");
  if (packed_bytes < q.bytes)
    return fail(RPD_ERR_WORKSPACE_TOO_SMALL, "packed has %zu bytes, %zu needed", packed_bytes, q.bytes);
  const hipError_t e = rpd::launch_quant_pack(q, codes, static_cast<const uint16_t*>(scales), zeros,
                                              static_cast<char*>(packed), static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

size_t rpd_quant_workspace_size(const rpd_quant_head* h, int32_t M, int32_t statistics) {
  if (!h || !quant_ok(h) || M < 1 || M > 1 << 20) return 0;
  rpd::QuantCall a{};
  a.M = M;
  a.stats = statistics != 0;
  const rpd::QuantDims q = quant_dims(h);
  quant_plan(q, a);
  return quant_space(q, a).bytes;
}

rpd_status rpd_quant_project(const rpd_quant_head* h, const void* packed, int32_t M, const void* x, int64_t x_stride,
                             void* logits, int64_t logits_stride, int32_t logits_dtype, int32_t* argmax,
                             float* confidence, float* entropy, float logit_scale, void* workspace,
                             size_t workspace_bytes, void* stream) {
  rpd::clear_error();
  rpd_status st = check_head(h);
  if (st != RPD_OK) return st;
  if (M < 0 || M > 1 << 20) return fail(RPD_ERR_BAD_SHAPE, "need 0<=M<=2^20 (got %d)", M);
  const int ns = (argmax != nullptr) + (confidence != nullptr) + (entropy != nullptr);
  if (x_stride < h->d || (logits && logits_stride < h->V))
    return fail(RPD_ERR_BAD_SHAPE, "row strides must be at least the row's length");
  if (logits && logits_dtype != h->dtype && logits_dtype != RPD_DTYPE_F32)
    return fail(RPD_ERR_UNSUPPORTED, "logits_dtype must be the head's or fp32 (got %d)", logits_dtype);
  if (!scale_ok(logit_scale))
    return fail(RPD_ERR_BAD_PARAM, "logit_scale must be finite and > 0, or 0 for 1 (got %g)", logit_scale);
  if (M == 0) return RPD_OK;
  if (!packed || !x) return fail(RPD_ERR_NULL_POINTER, "packed and x are required");
  if (logits ? ns != 0 : ns != 3)
    return fail(RPD_ERR_NULL_POINTER, "give either logits, or argmax, confidence and entropy");
  if (misaligned(packed, 255)) return fail(RPD_ERR_UNSUPPORTED, "packed must be 256-byte aligned");
  if (misaligned(x, 1) || misaligned(logits, elem_align(logits_dtype)) || misaligned(argmax, 3) ||
      misaligned(confidence, 3) || misaligned(entropy, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  const rpd::QuantDims q = quant_dims(h);
  const char* pk = static_cast<const char*>(packed);
  rpd::QuantCall a{};
  a.codes = reinterpret_cast<const rpd::codes_t*>(pk);
  a.scales = reinterpret_cast<const uint16_t*>(pk + q.scale_offset);
  a.zeros = h->has_zeros ? reinterpret_cast<const uint8_t*>(pk + q.zero_offset) : nullptr;
  a.x = static_cast<const uint16_t*>(x);
  a.x_stride = x_stride;
  a.x_vec = !misaligned(x, 15) && (M == 1 || x_stride % 8 == 0);
  a.bf16 = h->dtype == RPD_DTYPE_BF16;
  a.M = M;
  a.stats = logits == nullptr;
  a.out = logits;
  a.out_stride = logits_stride;
  a.out_type = logits_dtype;
  a.logit_scale = scale_of(logit_scale);
  a.argmax = argmax;
  a.confidence = confidence;
  a.entropy = entropy;
  quant_plan(q, a);
  const QuantSpace w = quant_space(q, a);
  if (w.bytes > 0) {
    st = check_workspace(workspace, workspace_bytes, w.bytes);
    if (st != RPD_OK) return st;
    char* ws = static_cast<char*>(workspace);
    if (M > 16) {
      a.xrows = reinterpret_cast<rpd::codes_t*>(ws);
      a.xexp = reinterpret_cast<int32_t*>(ws + w.exps);
    }
    a.partials = reinterpret_cast<float4*>(ws + w.states);
  }
  const hipError_t e = rpd::launch_quant_project(q, a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

size_t rpd_verify_workspace_size(const rpd_verify* p) {
  if (!p || !verify_shape_ok(p)) return 0;
  return verify_plan(p).bytes;
}

rpd_status rpd_verify_draft(const rpd_verify* p, void* workspace, size_t workspace_bytes, void* stream) {
  rpd::clear_error();
  if (!p) return fail(RPD_ERR_NULL_POINTER, "problem is NULL");
  if (!verify_shape_ok(p))
    return fail(RPD_ERR_BAD_SHAPE, "need B>=1, T>=0, B*(T+1)<=2^20, 1<=V<=2^28 (got B=%d T=%d V=%d)", p->B, p->T, p->V);
  if (!is_float_dtype(p->dtype)) return fail(RPD_ERR_UNSUPPORTED, "dtype %d is not supported", p->dtype);
  if (p->flags & ~RPD_VERIFY_GREEDY) return fail(RPD_ERR_BAD_PARAM, "flags holds unknown bits (0x%x)", p->flags);
  const bool greedy = (p->flags & RPD_VERIFY_GREEDY) != 0;
  if (!greedy && (!scale_ok(p->target_scale) || !scale_ok(p->draft_scale)))
    return fail(RPD_ERR_BAD_PARAM, "target_scale and draft_scale must be finite and > 0, or 0 for 1 (got %g, %g)",
                p->target_scale, p->draft_scale);
  if (!p->target || !p->out_token || !p->n_accept)
    return fail(RPD_ERR_NULL_POINTER, "target, out_token and n_accept are required");
  if (p->T > 0 && (!p->token || !p->accept)) return fail(RPD_ERR_NULL_POINTER, "token and accept are required");
  if (!greedy && (!p->r || (p->T > 0 && !p->u))) return fail(RPD_ERR_NULL_POINTER, "u and r are required");
  // rows of one sequence, and sequences, may be laid out in any order, also overlapping: they are only read
  if (p->target_batch_stride < 0 || p->target_row_stride < 0 || p->draft_batch_stride < 0 || p->draft_row_stride < 0)
    return fail(RPD_ERR_BAD_SHAPE, "strides must be >= 0");
  const unsigned e_al = elem_align(p->dtype);
  if (misaligned(p->target, e_al) || misaligned(p->draft, e_al) || misaligned(p->token, 3) || misaligned(p->len, 3) ||
      misaligned(p->u, 3) || misaligned(p->r, 3) || misaligned(p->out_token, 3) || misaligned(p->n_accept, 3) ||
      misaligned(p->accept, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  const VerifyPlan v = verify_plan(p);
  if (v.rows * v.splits > kMaxBlocks) return fail(RPD_ERR_BAD_SHAPE, "B * T * V is too large");
  rpd_status st = check_workspace(workspace, workspace_bytes, v.bytes);
  if (st != RPD_OK) return st;
  rpd::VerifyCall a{};
  a.B = p->B;
  a.T = p->T;
  a.V = p->V;
  a.dtype = p->dtype;
  a.target = p->target;
  a.t_batch = p->target_batch_stride;
  a.t_row = p->target_row_stride;
  a.draft = greedy ? nullptr : p->draft;
  a.d_batch = p->draft_batch_stride;
  a.d_row = p->draft_row_stride;
  a.token = p->token;
  a.len = p->len;
  a.u = p->u;
  a.r = p->r;
  a.target_scale = scale_of(p->target_scale);
  a.draft_scale = scale_of(p->draft_scale);
  a.greedy = greedy;
  a.out_token = p->out_token;
  a.n_accept = p->n_accept;
  a.accept = p->accept;
  char* ws = static_cast<char*>(workspace);
  a.stats = reinterpret_cast<rpd::RowPart*>(ws);
  a.picks = reinterpret_cast<rpd::VerifyPick*>(ws + v.picks);
  a.sums = reinterpret_cast<double*>(ws + v.sums);
  a.totals = v.single ? reinterpret_cast<double*>(ws + v.totals) : nullptr;
  a.splits = v.splits;
  a.chunk = v.chunk;
  a.parts = v.parts;
  a.part = v.part;
  const hipError_t e = rpd::launch_verify(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

size_t rpd_distill_workspace_size(const rpd_distill* p) {
  if (!p || !distill_shape_ok(p) || p->N == 0) return 0;
  return distill_plan(p).bytes;
}

rpd_status rpd_distill_loss(const rpd_distill* p, void* workspace, size_t workspace_bytes, void* stream) {
  rpd::clear_error();
  rpd_status st = check_distill(p, p && p->grad != nullptr);
  if (st != RPD_OK) return st;
  if (p->N == 0) return RPD_OK;
  if (!p->loss) return fail(RPD_ERR_NULL_POINTER, "loss is required");
  st = check_workspace(workspace, workspace_bytes, distill_plan(p).bytes);
  if (st != RPD_OK) return st;
  const hipError_t e = rpd::launch_distill_loss(distill_call(p, workspace), static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

rpd_status rpd_distill_grad(const rpd_distill* p, void* stream) {
  rpd::clear_error();
  rpd_status st = check_distill(p, true);
  if (st != RPD_OK) return st;
  if (p->N == 0) return RPD_OK;
  const hipError_t e = rpd::launch_distill_grad(distill_call(p, nullptr), static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

}  // extern "C"
