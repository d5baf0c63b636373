// C ABI of the 8-bit floating-point blocks: argument validation, workspace
// layout and launch planning. Kernels live in fp8.hip.
#include <algorithm>

#include "rpd_checks.h"

using namespace rpd;

namespace {

bool head_ok(int V, int d) { return V >= 1 && V <= 1 << 20 && d >= 1 && d <= 1 << 20 && (long long)V * d <= 1LL << 35; }

rpd_status check_head(int V, int d) {
  if (!head_ok(V, d)) return fail(RPD_ERR_BAD_SHAPE, "need 1<=V,d<=2^20, V*d<=2^35 (got V=%d d=%d)", V, d);
  return RPD_OK;
}

// Rows that the launches hold: at most (V / 256 + 8) (M / 128 + 2) workgroups for the tiles of a whole sum and (M / 16 + 1)
// (d / 512 + 1) for the rows, below 2^24 each. (Sums that are cut along the columns have fewer than 512 tiles.)
bool rows_ok(int V, int d, int M) {
  return M >= 1 && M <= 1 << 20 && (long long)M * V <= 1LL << 38 && (long long)M * d <= 1LL << 36;
}

Fp8Dims fp8_dims(int V, int d) {
  Fp8Dims q{};
  q.V = V;
  q.d = d;
  q.nc = (int)up_div(d, kFp8Block);
  q.n16 = (int)up_div(V, 16);
  q.nr = (int)up_div(V, kFp8Block);
  q.scale_offset = round256((size_t)q.n16 * q.nc * 2048);
  q.bytes = q.scale_offset + round256((size_t)q.nr * q.nc * 4);
  return q;
}

constexpr int kWanted = 512;      // workgroups: two on each of 256 CUs
constexpr int kLeastChunks = 4;   // of a split

// Up to as many rows, the workgroups quantize them themselves: 126464 x 4096, bf16, one row 80 us so and 84 laid out
// first, 16 rows 82 and 86; 32 rows 90 and 88.
constexpr int kOwnRows = 16;

void fp8_plan(const Fp8Dims& q, Fp8Call& a) {
  // As few tiles as 8 blocks of rows allow (no more fit the registers), all of about one size: 1024 rows of 126464 x 4096
  // 850 us so, 910 in tiles of up to 6 blocks, 963 of up to 4.
  a.mb = (int)up_div(a.M, 16);
  a.nrt = (int)up_div(a.mb, kFp8TileBlocks);
  a.nb = (int)up_div(a.mb, a.nrt);
  a.nrt = (int)up_div(a.mb, a.nb);
  a.nvt = (int)up_div(q.V, kFp8TileRows);
  // a small head is cut along its columns as well, the parts' sums joined in order
  a.splits = 1;
  const long long tiles = (long long)a.nrt * a.nvt;
  if (tiles < kWanted)
    a.splits = (int)std::max(1LL, std::min(kWanted / tiles, (long long)q.nc / kLeastChunks));
  // Where a last round after full ones has at most a quarter of the workgroups that run at a time, its tiles are cut into as
  // many pieces as fit one (a launch of its own, so of little use to more): 152064 x 3584, bf16, 64 rows 120 us so and 132
  // in whole tiles, 101 rows 156 and 164, 128 rows 164 and 175; 256 rows, with a third of a round left, 292 and 274.
  a.vt0 = a.nvt;
  const long long jobs = tiles * a.splits, rest = jobs % kWanted;
  if (a.nb >= 4 && jobs > kWanted && rest > 0 && rest <= kWanted / 4) {
    a.vt0 = (int)((jobs - rest) / a.nrt);
    const int pieces = std::max(1, kWanted / (a.nvt - a.vt0));
    a.last_nb = std::min(a.nb, (int)up_div(a.mb, pieces));
    if (a.last_nb == a.nb) a.vt0 = a.nvt;
  }
}

struct Fp8Space {
  size_t partials, sums, bytes;   // offsets (the rows come first)
};
Fp8Space fp8_space(const Fp8Dims& q, const Fp8Call& a, bool stats) {
  Fp8Space w{};
  w.partials = a.M > kOwnRows ? round256((size_t)a.mb * q.nc * 4096) : 0;
  w.sums = w.partials + (stats && a.splits == 1 ? round256((size_t)a.M * a.nvt * 16) : 0);
  w.bytes = w.sums + (a.splits > 1 ? round256((size_t)a.splits * a.M * q.n16 * 64) : 0);
  return w;
}

}  // namespace

extern "C" {

rpd_status rpd_fp8_quantize(int32_t rows, int32_t d, int32_t dtype, const void* x, int64_t x_stride, int32_t block_rows,
                            uint8_t* codes, int64_t codes_stride, float* scales, void* stream) {
  clear_error();
  if (rows < 0 || rows > 1 << 28 || d < 1 || d > 1 << 28)
    return fail(RPD_ERR_BAD_SHAPE, "need 0<=rows<=2^28, 1<=d<=2^28 (got rows=%d d=%d)", rows, d);
  if (!is_float_dtype(dtype)) return fail(RPD_ERR_UNSUPPORTED, "dtype %d is not supported", dtype);
  if (block_rows != 1 && block_rows != kFp8Block)
    return fail(RPD_ERR_BAD_PARAM, "block_rows must be 1 or %d (got %d)", kFp8Block, block_rows);
  if (x_stride < d || codes_stride < d) return fail(RPD_ERR_BAD_SHAPE, "row strides must be at least d");
  const long long nb = up_div(d, kFp8Block);
  if ((block_rows == 1 ? up_div(rows * nb, 16) : up_div(rows, kFp8Block) * nb) > kMaxBlocks)
    return fail(RPD_ERR_BAD_SHAPE, "rows * d is too large (rows=%d d=%d)", rows, d);
  if (rows == 0) return RPD_OK;
  if (!x || !codes || !scales) return fail(RPD_ERR_NULL_POINTER, "x, codes and scales are required");
  if (misaligned(x, elem_align(dtype)) || misaligned(scales, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  // what is written must not be what other workgroups still read
  const long long xs = x_stride * size_of(dtype), xn = (long long)d * size_of(dtype), span_x = (rows - 1) * xs + xn,
                  span_c = (rows - 1) * codes_stride + d,
                  sn = (block_rows == 1 ? rows : up_div(rows, kFp8Block)) * nb * 4;
  if (rows_meet(x, xs, xn, codes, codes_stride, d, rows) || rows_meet(x, 0, span_x, scales, 0, sn, 1) ||
      rows_meet(codes, 0, span_c, scales, 0, sn, 1))
    return fail(RPD_ERR_BAD_PARAM, "x, codes and scales must not overlap");
  Fp8Quantize a{};
  a.rows = rows;
  a.d = d;
  a.nb = (int)nb;
  a.dtype = dtype;
  a.x = x;
  a.x_stride = x_stride;
  a.codes = codes;
  a.codes_stride = codes_stride;
  a.scales = scales;
  const hipError_t e = launch_fp8_quantize(a, block_rows, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

size_t rpd_fp8_packed_size(int32_t V, int32_t d) { return head_ok(V, d) ? fp8_dims(V, d).bytes : 0; }

rpd_status rpd_fp8_pack(int32_t V, int32_t d, const uint8_t* codes, const float* scales, int32_t transpose, void* packed,
                        size_t packed_bytes, void* stream) {
  clear_error();
  const rpd_status st = check_head(V, d);
  if (st != RPD_OK) return st;
  if (transpose != 0 && transpose != 1) return fail(RPD_ERR_BAD_PARAM, "transpose must be 0 or 1");
  if (!codes || !scales || !packed) return fail(RPD_ERR_NULL_POINTER, "codes, scales and packed are required");
  if (misaligned(scales, 3)) return fail(RPD_ERR_UNSUPPORTED, "scales must be aligned to their element");
  if (misaligned(packed, 255)) return fail(RPD_ERR_UNSUPPORTED, "packed must be 256-byte aligned");
  const Fp8Dims q = transpose ? fp8_dims(d, V) : fp8_dims(V, d);
  if (packed_bytes < q.bytes)
    return fail(RPD_ERR_WORKSPACE_TOO_SMALL, "packed has %zu bytes, %zu needed", packed_bytes, q.bytes);
  const long long bytes = (long long)q.bytes;
  if (rows_meet(codes, 0, (long long)V * d, packed, 0, bytes, 1) ||
      rows_meet(scales, 0, up_div(V, kFp8Block) * up_div(d, kFp8Block) * 4, packed, 0, bytes, 1))
    return fail(RPD_ERR_BAD_PARAM, "packed must not overlap codes or scales");   // both are read while it is written
  const hipError_t e =
      launch_fp8_pack(q, codes, scales, transpose != 0, static_cast<uint8_t*>(packed), static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

size_t rpd_fp8_workspace_size(int32_t V, int32_t d, int32_t M, int32_t statistics) {
  if (!head_ok(V, d) || !rows_ok(V, d, M)) return 0;
  const Fp8Dims q = fp8_dims(V, d);
  Fp8Call a{};
  a.M = M;
  fp8_plan(q, a);
  return fp8_space(q, a, statistics != 0).bytes;
}

rpd_status rpd_fp8_project(int32_t V, int32_t d, const void* packed, int32_t M, const void* x, int64_t x_stride,
                           int32_t x_dtype, void* logits, int64_t logits_stride, int32_t logits_dtype, int32_t* argmax,
                           float* confidence, float* entropy, float logit_scale, void* workspace, size_t workspace_bytes,
                           void* stream) {
  clear_error();
  rpd_status st = check_head(V, d);
  if (st != RPD_OK) return st;
  if (M < 0 || M > 1 << 20) return fail(RPD_ERR_BAD_SHAPE, "need 0<=M<=2^20 (got %d)", M);
  if (!is_float_dtype(x_dtype)) return fail(RPD_ERR_UNSUPPORTED, "x_dtype %d is not supported", x_dtype);
  if (x_stride < d || (logits && logits_stride < V))
    return fail(RPD_ERR_BAD_SHAPE, "row strides must be at least the row's length");
  if (logits && !is_float_dtype(logits_dtype))
    return fail(RPD_ERR_UNSUPPORTED, "logits_dtype %d is not supported", logits_dtype);
  if (!scale_ok(logit_scale))
    return fail(RPD_ERR_BAD_PARAM, "logit_scale must be finite and > 0, or 0 for 1 (got %g)", logit_scale);
  if (M == 0) return RPD_OK;
  if (!rows_ok(V, d, M))
    return fail(RPD_ERR_BAD_SHAPE, "need M*V<=2^38, M*d<=2^36 (got M=%d V=%d d=%d)", M, V, d);
  if (!packed || !x) return fail(RPD_ERR_NULL_POINTER, "packed and x are required");
  const int ns = (argmax != nullptr) + (confidence != nullptr) + (entropy != nullptr);
  if (logits ? ns != 0 : ns != 3)
    return fail(RPD_ERR_NULL_POINTER, "give either logits, or argmax, confidence and entropy");
  if (misaligned(packed, 255)) return fail(RPD_ERR_UNSUPPORTED, "packed must be 256-byte aligned");
  if (misaligned(x, elem_align(x_dtype)) || misaligned(logits, elem_align(logits_dtype)) || misaligned(argmax, 3) ||
      misaligned(confidence, 3) || misaligned(entropy, 3))
    return fail(RPD_ERR_UNSUPPORTED, "a pointer is not aligned to its element");
  const int xb = size_of(x_dtype), ob = size_of(logits_dtype);
  if (logits && rows_meet(x, x_stride * xb, (long long)d * xb, logits, logits_stride * ob, (long long)V * ob, M))
    return fail(RPD_ERR_BAD_PARAM, "logits must not overlap x");   // workgroups read x while others write
  const Fp8Dims q = fp8_dims(V, d);
  const uint8_t* pk = static_cast<const uint8_t*>(packed);
  Fp8Call a{};
  a.packed = pk;
  a.scales = reinterpret_cast<const float*>(pk + q.scale_offset);
  a.M = M;
  a.x = x;
  a.x_stride = x_stride;
  a.x_type = x_dtype;
  a.out = logits;
  a.out_stride = logits_stride;
  a.out_type = logits_dtype;
  a.logit_scale = scale_of(logit_scale);
  a.argmax = argmax;
  a.confidence = confidence;
  a.entropy = entropy;
  fp8_plan(q, a);
  const Fp8Space w = fp8_space(q, a, logits == nullptr);
  if (w.bytes > 0) {
    st = check_workspace(workspace, workspace_bytes, w.bytes);
    if (st != RPD_OK) return st;
    char* ws = static_cast<char*>(workspace);
    a.xrows = M > kOwnRows ? reinterpret_cast<uint8_t*>(ws) : nullptr;
    a.partials = reinterpret_cast<float4*>(ws + w.partials);
    a.sums = reinterpret_cast<float*>(ws + w.sums);
  }
  const hipError_t e = launch_fp8_project(q, a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RPD_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return RPD_OK;
}

}  // extern "C"
