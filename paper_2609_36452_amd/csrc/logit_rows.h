// Device pieces shared by the kernels that read rows of logits from memory:
// eight elements of a row at a time, whatever its alignment, and running
// softmax sums.
#pragma once

#include <cmath>
#include <cstdint>

#include "rpd_device.h"

namespace rpd {
namespace {

// Rows of an odd length start at any element; wide global loads and stores
// need no alignment beyond the element's here.
struct __attribute__((packed, aligned(2))) Any16 {
  u32x4 v;
};
struct __attribute__((packed, aligned(4))) Any32 {
  u32x4 a, b;
};

struct Bf16 {
  typedef uint16_t t;
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ t to(float x) { return __builtin_bit_cast(t, (__bf16)x); }
};
struct F16 {
  typedef uint16_t t;
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const t* p) { return (float)__builtin_bit_cast(_Float16, *p); }
  static __device__ __forceinline__ t to(float x) { return __builtin_bit_cast(t, (_Float16)x); }
};
struct F32 {
  typedef float t;
  static constexpr int bytes = 4;
  static __device__ __forceinline__ float one(const t* p) { return *p; }
  static __device__ __forceinline__ t to(float x) { return x; }
};

// eight elements as they lie in memory
template <class E>
struct Eight {
  u32x4 v;
  __device__ __forceinline__ void load(const typename E::t* p) { v = reinterpret_cast<const Any16*>(p)->v; }
  // past the caches
  __device__ __forceinline__ void stream(typename E::t* p) const {
    __builtin_nontemporal_store(v, &reinterpret_cast<Any16*>(p)->v);
  }
  __device__ __forceinline__ float at(int e) const;
  __device__ __forceinline__ void set(const float (&z)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (uint32_t)E::to(z[2 * e]) | (uint32_t)E::to(z[2 * e + 1]) << 16;
  }
};
template <>
__device__ __forceinline__ float Eight<Bf16>::at(int e) const {
  const uint32_t w = v[e >> 1];
  return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
}
template <>
__device__ __forceinline__ float Eight<F16>::at(int e) const {
  const uint32_t w = v[e >> 1];
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(e & 1 ? w >> 16 : w));
}
template <>
struct Eight<F32> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const Any32*>(p)->a;
    b = reinterpret_cast<const Any32*>(p)->b;
  }
  __device__ __forceinline__ void stream(float* p) const {
    __builtin_nontemporal_store(a, &reinterpret_cast<Any32*>(p)->a);
    __builtin_nontemporal_store(b, &reinterpret_cast<Any32*>(p)->b);
  }
  __device__ __forceinline__ float at(int e) const { return __uint_as_float(e < 4 ? a[e & 3] : b[e & 3]); }
  __device__ __forceinline__ void set(const float (&z)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = __float_as_uint(z[e]);
      b[e] = __float_as_uint(z[4 + e]);
    }
  }
};

// 8 entries of a row from i on, -inf past `hi`
template <class E>
__device__ __forceinline__ void load_eight(const typename E::t* p, int i, int hi, Eight<E>& v) {
  if (i + 8 <= hi) {
    v.load(p + i);
  } else {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = i + e < hi ? E::one(p + i + e) : -INFINITY;
    v.set(z);
  }
}

// Maximum m of the raw logits and S = sum e^(scale (z - m)). Nothing seen: m =
// -inf, S = 0; a row that is -inf throughout keeps S = 0; NaN and +inf leave S
// NaN.
struct MaxSum {
  float m, S;
};
// what exponents are relative to
__device__ __forceinline__ float top_of(float m) { return m == -INFINITY ? 0.f : m; }
// e^(scale (z - top)) for z up to top. The difference first: scale * top may be above float32's range though z and top
// are not, and where it is not, its rounding alone may be more than any exponent (a mask of the type's lowest value).
// The two roundings are 2^-24 of the exponent each.
__device__ __forceinline__ float exp_below(float z, float top, float scale) { return __expf((z - top) * scale); }
// what a sum relative to m is worth relative to `top` (0 while nothing was seen)
__device__ __forceinline__ float carry(float m, float top, float scale) {
  return m == -INFINITY ? 0.f : exp_below(m, top, scale);
}

}  // namespace
}  // namespace rpd
