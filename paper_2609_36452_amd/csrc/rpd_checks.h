// Argument checks shared by the C entries of the operators around the commit
// step (host code).
#pragma once

#include <cmath>

#include "rpd_ops.h"

namespace rpd {
namespace {

constexpr long long kMaxBlocks = (1LL << 24) - 1;   // workgroups of 256 threads: a launch holds fewer than 2^32 threads

bool is_float_dtype(int t) { return t == RPD_DTYPE_BF16 || t == RPD_DTYPE_F16 || t == RPD_DTYPE_F32; }
unsigned elem_align(int t) { return t == RPD_DTYPE_F32 ? 3u : 1u; }
bool misaligned(const void* p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }
long long up_div(long long a, long long b) { return (a + b - 1) / b; }

// an inverse temperature: 0 is read as 1
bool scale_ok(float s) { return std::isfinite(s) && s >= 0.f; }
float scale_of(float s) { return s == 0.f ? 1.f : s; }

rpd_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return fail(RPD_ERR_NULL_POINTER, "workspace is NULL (%zu bytes needed)", need);
  if (misaligned(ws, 255)) return fail(RPD_ERR_UNSUPPORTED, "workspace must be 256-byte aligned");
  if (have < need) return fail(RPD_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", have, need);
  return RPD_OK;
}

}  // namespace
}  // namespace rpd
