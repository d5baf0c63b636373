// Argument checks shared by the C entries of the operators around the commit
// step (host code).
#pragma once

#include <cmath>
#include <cstdint>

#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr long long kMaxBlocks = (1LL << 24) - 1;   // workgroups of 256 threads: a launch holds fewer than 2^32 threads

bool is_float_dtype(int t) { return t == RPD_DTYPE_BF16 || t == RPD_DTYPE_F16 || t == RPD_DTYPE_F32; }
unsigned elem_align(int t) { return t == RPD_DTYPE_F32 ? 3u : 1u; }
bool misaligned(const void* p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }
int size_of(int t) { return t == RPD_DTYPE_F32 ? 4 : 2; }
long long up_div(long long a, long long b) { return (a + b - 1) / b; }

// an inverse temperature: 0 is read as 1
bool scale_ok(float s) { return std::isfinite(s) && s >= 0.f; }
float scale_of(float s) { return s == 0.f ? 1.f : s; }

// Whether rows of pn bytes, ps apart from p on, and as many of qn bytes, qs apart from q on, may have a byte in common:
// those of one stride may lie between each other; of two strides, the ranges must be apart.
bool rows_meet(const void* p, long long ps, long long pn, const void* q, long long qs, long long qn, long long rows) {
  const __int128 at = (__int128) reinterpret_cast<uintptr_t>(q) - (__int128) reinterpret_cast<uintptr_t>(p);
  if (at >= (__int128)(rows - 1) * ps + pn || -at >= (__int128)(rows - 1) * qs + qn) return false;
  if (rows == 1 || ps != qs) return true;
  const long long shift = (long long)(((at % ps) + ps) % ps);
  return shift < pn || shift > ps - qn;
}

rpd_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return fail(RPD_ERR_NULL_POINTER, "workspace is NULL (%zu bytes needed)", need);
  if (misaligned(ws, 255)) return fail(RPD_ERR_UNSUPPORTED, "workspace must be 256-byte aligned");
  if (have < need) return fail(RPD_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", have, need);
  return RPD_OK;
}

}  // namespace
}  // namespace rpd
