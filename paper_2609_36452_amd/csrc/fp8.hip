// Blocks of 8-bit floating point (e4m3, a scale for each block of 128), and
// an output head of them.
//
//   quantization: of a block of 128 columns of a row, or of 128 x 128 of a
//   matrix, scale = the smallest power of two with max |x| <= 448 scale, code
//   = e4m3(x / scale). The division is exact, so a code is rounded once.
//   head: y[m][v] = sum over blocks b of columns of
//         scale[v / 128][b] * sum_k code[v][k] x^[m][k]
//   with x^ the row's quantized values. The rows' scales are powers of two, so
//   x^ is a bf16 number; the head's are any float32, so they multiply each
//   block's sum in float32.
//
// The products run on the bf16 matrix cores, codes converted in registers:
// operands exact, sums float32. (The 8-bit matrix instructions add the
// products of an instruction in a window of fewer bits than float32: off by
// 1.4e-5 of the sum's size for Gaussian rows, 8e-5 with one large entry in a
// block, where the bf16 ones are off by 1e-8 to 7e-8. That is too much for
// float32 logits and for the statistics.)
#include <cstdint>
#include <type_traits>

#include "logit_rows.h"
#include "reduce_device.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(1))) Any8 {   // codes: eight bytes anywhere
  u32x2 v;
};
struct __attribute__((packed, aligned(1))) Bytes16 {
  u32x4 v;
};
struct __attribute__((packed, aligned(2))) Half4 {   // four 16-bit logits at any element
  u32x2 v;
};
struct __attribute__((packed, aligned(4))) Float4 {
  f32x4 v;
};

constexpr int kBlock = kFp8Block;

// ---------------------------------------------------------- quantization --

// the largest finite magnitude of eight entries
__device__ __forceinline__ float top_of_eight(const float (&z)[8]) {
  float t = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = fabsf(z[e]);
    t = fmaxf(t, a < INFINITY ? a : 0.f);
  }
  return t;
}

// The scale 2^e of a block from its largest magnitude 1.m 2^x, by the bits:
// 448 is 1.75 2^8, so e is x - 8, and one more where 1.m is above 1.75. e
// stays within -126 .. 120, so the scale and its inverse are normal numbers; a
// block of zeros has scale 1.
__device__ __forceinline__ float scale_of_top(float top) {
  if (top == 0.f) return 1.f;
  const uint32_t b = __float_as_uint(top);
  const int e = max((int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float inverse_of_power(float s) {
  return __uint_as_float(0x7f000000u - __float_as_uint(s));   // 2^-e
}

// codes of eight entries; what is not finite becomes NaN
__device__ __forceinline__ u32x2 codes_of_eight(const float (&z)[8], float inv) {
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = fabsf(z[e]) < INFINITY ? z[e] * inv : NAN;
  u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], 0, false);
    r[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], w, true);
  }
  return r;
}

// eight entries of a row of d from k on, 0 past its end (p: the row, or NULL for a row of zeros)
template <class E>
__device__ __forceinline__ void row_eight(const typename E::t* p, int k, int d, float (&z)[8]) {
  Eight<E> v;
  if (p && k < d) load_eight<E>(p, k, d, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = p && k + e < d ? v.at(e) : 0.f;
}

__device__ __forceinline__ void store_codes(uint8_t* p, int k, int d, const u32x2 c) {
  if (k + 8 <= d) {
    reinterpret_cast<Any8*>(p + k)->v = c;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < d) p[k + e] = (uint8_t)(c[e >> 2] >> (8 * (e & 3)));
  }
}

// 16 lanes a block of a row, 8 entries each, held between the maximum and the codes: 13 x 3584 fp16 takes 2.8 us. Many rows
// are bound by memory: 65536 x 4096 takes 163 us of bf16 and of fp16 (5.0 TB/s), 227 of fp32 (5.9), 8192 rows 21 and 25.
template <class E>
__global__ __launch_bounds__(256) void k_fp8_quantize_rows(Fp8Quantize a) {
  const long long g = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int i = threadIdx.x & 15;
  if (g >= (long long)a.rows * a.nb) return;   // whole groups of 16 lanes
  const int row = (int)(g / a.nb), b = (int)(g - (long long)row * a.nb);
  float z[8];
  row_eight<E>(static_cast<const typename E::t*>(a.x) + row * a.x_stride, b * kBlock + 8 * i, a.d, z);
  float top = top_of_eight(z);
#pragma unroll
  for (int k = 8; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
  const float s = scale_of_top(top);
  store_codes(a.codes + row * a.codes_stride, b * kBlock + 8 * i, a.d, codes_of_eight(z, inverse_of_power(s)));
  if (i == 0) a.scales[g] = s;
}

// a workgroup a block of 128 x 128, 64 entries a thread held in registers, so that memory is read once: bound by it, 126464
// x 4096 bf16 (1.55 GB read and written) takes 300 us, 5.2 TB/s
template <class E>
__global__ __launch_bounds__(256) void k_fp8_quantize_blocks(Fp8Quantize a) {
  const int rb = blockIdx.x / a.nb, b = blockIdx.x - rb * a.nb;
  const int r = threadIdx.x >> 4, k = b * kBlock + 8 * (threadIdx.x & 15);
  __shared__ float s_top[4];
  Eight<E> held[8];
  auto row_at = [&](int j) { return rb * kBlock + 16 * j + r; };
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (row_at(j) < a.rows && k < a.d)
      load_eight<E>(static_cast<const typename E::t*>(a.x) + row_at(j) * a.x_stride, k, a.d, held[j]);
  auto get = [&](int j, float (&z)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = row_at(j) < a.rows && k + e < a.d ? held[j].at(e) : 0.f;
  };
  float top = 0.f, z[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    get(j, z);
    top = fmaxf(top, top_of_eight(z));
  }
#pragma unroll
  for (int j = 32; j >= 1; j >>= 1) top = fmaxf(top, __shfl_xor(top, j));
  if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  const float s = scale_of_top(top), inv = inverse_of_power(s);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    get(j, z);
    if (row_at(j) < a.rows && k < a.d) store_codes(a.codes + row_at(j) * a.codes_stride, k, a.d, codes_of_eight(z, inv));
  }
  if (threadIdx.x == 0) a.scales[blockIdx.x] = s;
}

// ------------------------------------------------------------------ head --

// Layout of a head: tiles of 16 rows x 128 columns, 2 KB each, a row's tiles
// one after another. Lane l of the matrix product's operand holds row l % 16
// and the 32 columns from 32 (l / 16) on; the tile has the first 16 of every
// lane, then the other 16. The four products of a chunk take 8 each. Done once for a head: 126464 x 4096 in 185 us, its
// transpose (below) in 275.
__global__ __launch_bounds__(256) void k_fp8_pack(const uint8_t* codes, uint8_t* out, int V, int d, int nc, long long n) {
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;   // a piece of 16 columns
  if (at >= n) return;
  const int lane = (int)(at & 63), h = (int)(at >> 6 & 1);
  const long long tile = at >> 7;
  const int c = (int)(tile % nc), v = (int)(tile / nc) * 16 + (lane & 15);
  const int k = c * kBlock + 32 * (lane >> 4) + 16 * h;
  u32x4 r = {0u, 0u, 0u, 0u};
  if (v < V && k < d) {
    const uint8_t* p = codes + (long long)v * d + k;
    if (k + 16 <= d) {
      r = reinterpret_cast<const Bytes16*>(p)->v;
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (k + e < d) r[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
    }
  }
  *reinterpret_cast<u32x4*>(out + at * 16) = r;
}

// the same of the transposed head (rows k, columns v) by 128 x 128 blocks through LDS
__global__ __launch_bounds__(256) void k_fp8_pack_transposed(const uint8_t* codes, uint8_t* out, int V, int d, int nc) {
  // row v of the block in LDS at 132 v: a lane reads 16 rows of one column
  __shared__ __attribute__((aligned(4))) uint8_t s[kBlock * 132];
  const int c = blockIdx.x % nc, kb = blockIdx.x / nc, tid = threadIdx.x;   // block of columns (v), of rows (k)
  if (d % 4 == 0 && (reinterpret_cast<uintptr_t>(codes) & 3) == 0) {
#pragma unroll 8
    for (int i = tid; i < kBlock * 32; i += 256) {   // four columns at once
      const int v = c * kBlock + (i >> 5), k = kb * kBlock + 4 * (i & 31);
      reinterpret_cast<uint32_t*>(s)[(i >> 5) * 33 + (i & 31)] =
          v < V && k < d ? *reinterpret_cast<const uint32_t*>(codes + (long long)v * d + k) : 0;
    }
  } else {
    for (int i = tid; i < kBlock * kBlock; i += 256) {
      const int v = c * kBlock + (i >> 7), k = kb * kBlock + (i & 127);
      s[(i >> 7) * 132 + (i & 127)] = v < V && k < d ? codes[(long long)v * d + k] : 0;
    }
  }
  __syncthreads();
  const int rows16 = (d + 15) / 16;
  for (int i = tid; i < 8 * 128; i += 256) {   // 8 tiles of 16 rows, 128 pieces each
    const int lane = i & 63, h = i >> 6 & 1, t = kb * 8 + (i >> 7);
    if (t >= rows16) continue;
    const int r = 16 * (i >> 7) + (lane & 15), v0 = 32 * (lane >> 4) + 16 * h;
    u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e >> 2] |= (uint32_t)s[(v0 + e) * 132 + r] << (8 * (e & 3));
    *reinterpret_cast<u32x4*>(out + (((long long)t * nc + c) * 128 + (i & 127)) * 16) = w;
  }
}

__global__ __launch_bounds__(256) void k_fp8_pack_scales(const float* scales, float* out, int nr, int nc, int transpose) {
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;   // of the packed head: [nr][nc]
  if (at >= (long long)nr * nc) return;
  const int r = (int)(at / nc), c = (int)(at - (long long)r * nc);
  out[at] = transpose ? scales[(long long)c * nr + r] : scales[at];
}

// eight quantized entries as bf16 operands (4 significant bits times a power of two); the 16 lanes of a row's block
__device__ __forceinline__ u32x4 operands_of_eight(const float (&z)[8]) {
  float top = top_of_eight(z);
#pragma unroll
  for (int k = 8; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
  const float s = scale_of_top(top);
  const u32x2 c = codes_of_eight(z, inverse_of_power(s));
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    o[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[h], s, false));
    o[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[h], s, true));
  }
  return o;
}
// where they go in a block of 16 rows x 128 columns: columns 8 i .. of row r, lane quad i / 4, product i % 4
__device__ __forceinline__ int operand_at(int r, int i) { return (i & 3) * 1024 + ((i >> 2) * 16 + r) * 16; }

// Rows of x quantized, as bf16 operands: blocks of 16 rows x 128 columns, 4 KB
// each in the order of the four products, [block of rows][chunk]. Rows past
// the last are zeros.
constexpr int kRowChunks = 4;   // chunks a workgroup
template <class E>
__global__ __launch_bounds__(256) void k_fp8_rows(Fp8Dims q, Fp8Call a) {
  const int groups = (q.nc + kRowChunks - 1) / kRowChunks;
  const int mb = blockIdx.x / groups, c0 = (blockIdx.x - mb * groups) * kRowChunks;
  const int r = threadIdx.x >> 4, i = threadIdx.x & 15, m = mb * 16 + r;
  const typename E::t* p = m < a.M ? static_cast<const typename E::t*>(a.x) + m * a.x_stride : nullptr;
  float z[kRowChunks][8];
#pragma unroll
  for (int j = 0; j < kRowChunks; ++j) row_eight<E>(p, (c0 + j) * kBlock + 8 * i, q.d, z[j]);
#pragma unroll
  for (int j = 0; j < kRowChunks; ++j) {
    if (c0 + j >= q.nc) break;
    const u32x4 o = operands_of_eight(z[j]);
    *reinterpret_cast<u32x4*>(a.xrows + ((long long)mb * q.nc + c0 + j) * 4096 + operand_at(r, i)) = o;
  }
}

// A tile of 256 rows of the head (64 a wave) x 16 NB rows of x over a range of
// chunks. The head goes from memory into registers, a chunk ahead, and is
// converted there once (a wave has its rows for itself); x goes straight into
// LDS, which the four waves share, a chunk ahead in two stages. 64 head rows a
// wave, because each fragment of x read from LDS then serves four products.
//   Up to about 48 rows of x memory bounds it: 126464 x 4096 in 80 us for one
// row (6.5 TB/s), 82 for 32. At 1024 rows (845 us, 1.25 PFLOP/s) the matrix
// cores work 56% of the time and vector instructions take 44% of a SIMD's: half
// a one for a code, one for a result and chunk. In between, neither: 594 tiles
// of 112 rows x 3584 take 144, two workgroups a CU waiting for each other's
// chunks, and 512 at a time.
// NT: the head past the caches (nobody else reads this part of it): 82 against
// 90 us for 16 rows, 92 and 104 for 48, 130 and 136 for 112. E: the workgroup
// quantizes x itself (a single block of 16 rows: there is time for it beside
// the loads, while k_fp8_rows' launch and round trip cost 4 us of 85; of two
// blocks it costs 3 us more than it saves); else (void) x is laid out.
template <int NB, bool NT, class E>
__global__ __launch_bounds__(256, 2) void k_fp8_tile(Fp8Dims q, Fp8Call a) {
  __shared__ __attribute__((aligned(1024))) uint8_t sx0[NB * 4096], sx1[NB * 4096];
  int job = 0, vt = 0;
  if (!map_job(blockIdx.x, a.tiles, a.nrt * a.splits, 0, job, vt)) return;
  vt += a.vt0;
  const int rt = job % a.nrt, sp = job / a.nrt;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = (int)((long long)q.nc * sp / a.splits), c1 = (int)((long long)q.nc * (sp + 1) / a.splits);
  const int mb0 = rt * NB, v0 = vt * kFp8TileRows + 64 * wid;

  // both through buffer loads: the chunk's offset in a scalar register, no address registers. In place of tiles past the
  // head's and blocks past the rows' the last one is read again; what comes of it is not stored.
  auto resource = [](const uint8_t* p, long long bytes) {   // 2^28 at most: 8 blocks of 2^20 columns
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, (int)bytes, 0x00020000);
  };
  const long long wrow = (long long)q.nc * 2048, xrow = (long long)q.nc * 4096;
  const int w0 = min(v0 / 16, q.n16 - 1), w_last = min(q.n16 - 1 - w0, 3), x_last = min(a.mb - 1 - mb0, NB - 1);
  const __amdgpu_buffer_rsrc_t wrs = resource(a.packed + w0 * wrow, (w_last + 1) * wrow);
  constexpr bool kOwn = !std::is_void<E>::value;
  using X = std::conditional_t<kOwn, E, F32>;
  const __amdgpu_buffer_rsrc_t xrs =
      kOwn ? resource(nullptr, 0) : resource(a.xrows + mb0 * xrow, (x_last + 1) * xrow);
  const float* sc = a.scales + (long long)min(v0 / kBlock, q.nr - 1) * q.nc;
  const int wo = lane * 16, xo = threadIdx.x * 16;

  u32x4 raw[4][2];
  f32x4 acc[NB][4];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[j][u] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto load_w = [&](int c, int past) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        raw[u][h] = __builtin_amdgcn_raw_buffer_load_b128(wrs, (wo + past) + h * 1024, (min(u, w_last) * q.nc + c) * 2048,
                                                          NT ? 2 : 0);
  };
  auto load_x = [&](int c, int past, uint8_t* stage) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          xrs, (__attribute__((address_space(3))) void*)(stage + j * 4096 + wid * 1024), 16, xo + past,
          (min(j, x_last) * q.nc + c) * 4096, 0, 0);
  };
  // or a thread's 8 columns of a row of each block
  float own[kOwn ? NB : 1][8];
  auto fetch_x = [&](int c) {
    const int r = threadIdx.x >> 4, k = c * kBlock + 8 * (threadIdx.x & 15);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int m = (mb0 + j) * 16 + r;
      row_eight<X>(m < a.M ? static_cast<const typename X::t*>(a.x) + m * a.x_stride : nullptr, k, q.d, own[j]);
    }
  };
  auto store_x = [&](uint8_t* stage) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      *reinterpret_cast<u32x4*>(stage + j * 4096 + operand_at(threadIdx.x >> 4, threadIdx.x & 15)) = operands_of_eight(own[j]);
  };
  // what this wave has loaded has landed; then all waves' has. (A fence alone does not wait for loads into LDS.)
  auto landed = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // chunk c from its stage, while the next one is on its way
  auto chunk = [&](int c, const uint8_t* stage, uint8_t* next) {
    const float s = sc[c];
    bf16x8 wf[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        u32x4 o;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int w = (int)raw[u][t >> 1][2 * (t & 1) + h];
          o[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
          o[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
        }
        wf[u][t] = __builtin_bit_cast(bf16x8, o);
      }
    // behind the last chunk: past the resource's end, where nothing is fetched (a branch would cost 30 registers)
    const int past = c + 1 < c1 ? 0 : INT_MIN;
    if constexpr (kOwn) fetch_x(c + 1 < c1 ? c + 1 : q.nc);   // (zeros past the columns)
    else load_x(c + 1, past, next);
    load_w(c + 1, past);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (NB > 4) __builtin_amdgcn_sched_barrier(0);   // one block of rows at a time: no registers for the next one's
      bf16x8 xf[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) xf[t] = *reinterpret_cast<const bf16x8*>(stage + j * 4096 + t * 1024 + lane * 16);
      f32x4 part[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) part[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) part[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[u][t], xf[t], part[u], 0, 0, 0);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][u][e] = fmaf(s, part[u][e], acc[j][u][e]);
    }
    if constexpr (kOwn) store_x(next);
    landed();   // the next chunk's, and this stage is free
  };

  if (c0 < c1) {
    if constexpr (kOwn) fetch_x(c0);
    else load_x(c0, 0, sx0);
    load_w(c0, 0);
    if constexpr (kOwn) store_x(sx0);
    landed();
    int c = c0;
    for (; c + 2 <= c1; c += 2) {
      chunk(c, sx0, sx1);
      chunk(c + 1, sx1, sx0);
    }
    if (c < c1) chunk(c, sx0, sx1);
  }

  // lane l holds row (l % 16) of a block of x against rows 4 (l / 16) + e of a tile of the head
  const int m0 = mb0 * 16 + (lane & 15), vq = v0 + 4 * (lane >> 4);
  if (a.argmax && a.splits == 1) {
    float4 (*red)[NB * 16] = reinterpret_cast<float4 (*)[NB * 16]>(sx0);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float z[16];
      int vi[16];
      bool ok[16];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[4 * u + e] = acc[j][u][e] * a.logit_scale;
          vi[4 * u + e] = vq + 16 * u + e;
          ok[4 * u + e] = vi[4 * u + e] < q.V;
        }
      Soft st = soft_from_values(z, vi, ok);
      st = soft_merge(st, soft_shfl_xor(st, 16));
      st = soft_merge(st, soft_shfl_xor(st, 32));
      if (lane < 16) red[wid][j * 16 + lane] = soft_pack(st);
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t < NB * 16 && mb0 * 16 + t < a.M) {
      Soft st = soft_unpack(red[0][t]);
#pragma unroll
      for (int w = 1; w < 4; ++w) st = soft_merge(st, soft_unpack(red[w][t]));
      a.partials[(long long)(mb0 * 16 + t) * a.nvt + vt] = soft_pack(st);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int m = m0 + 16 * j;
    if (m >= a.M) continue;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int v = vq + 16 * u;
      if (v >= q.V) continue;
      if (a.splits > 1) {   // rows of the sums are padded to whole tiles
        *reinterpret_cast<f32x4*>(a.sums + ((long long)sp * a.M + m) * q.n16 * 16 + v) = acc[j][u];
        continue;
      }
      const long long at = m * a.out_stride + v;
      if (a.out_type == RPD_DTYPE_F32) {
        float* o = static_cast<float*>(a.out) + at;
        if (v + 4 <= q.V) {
          reinterpret_cast<Float4*>(o)->v = acc[j][u];
        } else {
          for (int e = 0; v + e < q.V; ++e) o[e] = acc[j][u][e];
        }
      } else {
        uint16_t* o = static_cast<uint16_t*>(a.out) + at;
        uint16_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = a.out_type == RPD_DTYPE_BF16 ? Bf16::to(acc[j][u][e]) : F16::to(acc[j][u][e]);
        if (v + 4 <= q.V) {
          reinterpret_cast<Half4*>(o)->v = u32x2{(uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16};
        } else {
          for (int e = 0; v + e < q.V; ++e) o[e] = h[e];
        }
      }
    }
  }
}

// the sums of the parts, in order (256 rows of 4096 from 2 parts: 12 us with its launch)
__global__ __launch_bounds__(256) void k_fp8_join(Fp8Dims q, Fp8Call a) {
  const int per = (q.V + 3) / 4;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  if (at >= (long long)a.M * per) return;
  const int m = (int)(at / per), v = 4 * (int)(at - (long long)m * per);
  const float* p = a.sums + (long long)m * q.n16 * 16 + v;
  const long long part = (long long)a.M * q.n16 * 16;
  f32x4 z = *reinterpret_cast<const f32x4*>(p);
  for (int s = 1; s < a.splits; ++s) z += *reinterpret_cast<const f32x4*>(p + s * part);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (v + e >= q.V) break;
    const long long o = m * a.out_stride + v + e;
    if (a.out_type == RPD_DTYPE_F32)
      static_cast<float*>(a.out)[o] = z[e];
    else
      static_cast<uint16_t*>(a.out)[o] = a.out_type == RPD_DTYPE_BF16 ? Bf16::to(z[e]) : F16::to(z[e]);
  }
}

// a workgroup a row: the same into its softmax statistics (a small head, whose tiles alone would not fill the GPU)
__global__ __launch_bounds__(256) void k_fp8_join_stats(Fp8Dims q, Fp8Call a) {
  __shared__ float4 s_wave[4];
  const int m = blockIdx.x, lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const float* p = a.sums + (long long)m * q.n16 * 16;
  const long long part = (long long)a.M * q.n16 * 16;
  Soft st = soft_empty();
  for (int v = 4 * threadIdx.x; v < q.V; v += 1024) {
    f32x4 y = *reinterpret_cast<const f32x4*>(p + v);
    for (int s = 1; s < a.splits; ++s) y += *reinterpret_cast<const f32x4*>(p + v + s * part);
    float z[4];
    int vi[4];
    bool ok[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] = y[e] * a.logit_scale;
      vi[e] = v + e;
      ok[e] = v + e < q.V;
    }
    st = soft_merge(st, soft_from_values(z, vi, ok));
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) st = soft_merge(st, soft_shfl_xor(st, k));
  if (lane == 0) s_wave[wid] = soft_pack(st);
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 4; ++w) st = soft_merge(st, soft_unpack(s_wave[w]));
    a.argmax[m] = st.idx == INT_MAX ? -1 : st.idx;
    a.confidence[m] = 1.f / st.S;
    a.entropy[m] = logf(st.S) - st.T / st.S;
  }
}

// one wave a row: the tiles' states -> argmax, top probability, entropy
__global__ __launch_bounds__(64) void k_fp8_stats(Fp8Call a) {
  const int m = blockIdx.x, lane = threadIdx.x;
  float4 keep[8];
  const Soft st = wave_merge_row(a.partials + (long long)m * a.nvt, a.nvt, lane, keep);
  if (lane == 0) {
    a.argmax[m] = st.idx == INT_MAX ? -1 : st.idx;   // a row of NaN has none
    a.confidence[m] = 1.f / st.S;
    a.entropy[m] = logf(st.S) - st.T / st.S;
  }
}

int tile_grid(const Fp8Call& a) { return 8 * ((a.tiles + 7) / 8) * a.nrt * a.splits; }

// more than 16 rows: tiles of 2 to 8 blocks of 16
template <int NB>
void tile_of(const Fp8Dims& q, const Fp8Call& a, hipStream_t s) {
  if (a.nrt == 1)
    k_fp8_tile<NB, true, void><<<tile_grid(a), 256, 0, s>>>(q, a);
  else
    k_fp8_tile<NB, false, void><<<tile_grid(a), 256, 0, s>>>(q, a);
}
void tile(const Fp8Dims& q, const Fp8Call& a, hipStream_t s) {
  switch (a.nb) {
    case 1: k_fp8_tile<1, false, void><<<tile_grid(a), 256, 0, s>>>(q, a); break;   // a last round's
    case 2: tile_of<2>(q, a, s); break;
    case 3: tile_of<3>(q, a, s); break;
    case 4: tile_of<4>(q, a, s); break;
    case 5: tile_of<5>(q, a, s); break;
    case 6: tile_of<6>(q, a, s); break;
    case 7: tile_of<7>(q, a, s); break;
    default: tile_of<8>(q, a, s); break;
  }
}
template <class E>
void own_tile(const Fp8Dims& q, const Fp8Call& a, hipStream_t s) {
  k_fp8_tile<1, true, E><<<tile_grid(a), 256, 0, s>>>(q, a);
}
template <class E>
void rows(const Fp8Dims& q, const Fp8Call& a, hipStream_t s) {
  k_fp8_rows<E><<<(unsigned)(a.mb * ((q.nc + kRowChunks - 1) / kRowChunks)), 256, 0, s>>>(q, a);
}

}  // namespace

hipError_t launch_fp8_quantize(const Fp8Quantize& a, int block_rows, hipStream_t s) {
  if (block_rows == 1) {
    const unsigned grid = (unsigned)(((long long)a.rows * a.nb + 15) / 16);
    if (a.dtype == RPD_DTYPE_BF16)
      k_fp8_quantize_rows<Bf16><<<grid, 256, 0, s>>>(a);
    else if (a.dtype == RPD_DTYPE_F16)
      k_fp8_quantize_rows<F16><<<grid, 256, 0, s>>>(a);
    else
      k_fp8_quantize_rows<F32><<<grid, 256, 0, s>>>(a);
  } else {
    const unsigned grid = (unsigned)(((a.rows + kBlock - 1) / kBlock) * a.nb);
    if (a.dtype == RPD_DTYPE_BF16)
      k_fp8_quantize_blocks<Bf16><<<grid, 256, 0, s>>>(a);
    else if (a.dtype == RPD_DTYPE_F16)
      k_fp8_quantize_blocks<F16><<<grid, 256, 0, s>>>(a);
    else
      k_fp8_quantize_blocks<F32><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_fp8_pack(const Fp8Dims& q, const uint8_t* codes, const float* scales, bool transpose, uint8_t* packed,
                           hipStream_t s) {
  if (transpose) {
    k_fp8_pack_transposed<<<(unsigned)(q.nr * q.nc), 256, 0, s>>>(codes, packed, q.d, q.V, q.nc);
  } else {
    const long long n = (long long)q.n16 * q.nc * 128;
    k_fp8_pack<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(codes, packed, q.V, q.d, q.nc, n);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long n = (long long)q.nr * q.nc;
  k_fp8_pack_scales<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(scales, reinterpret_cast<float*>(packed + q.scale_offset),
                                                               q.nr, q.nc, transpose);
  return hipGetLastError();
}

hipError_t launch_fp8_project(const Fp8Dims& q, const Fp8Call& a, hipStream_t s) {
  hipError_t e;
  Fp8Call whole = a;
  whole.vt0 = 0;
  whole.tiles = a.vt0;
  if (!a.xrows) {
    if (a.x_type == RPD_DTYPE_BF16)
      own_tile<Bf16>(q, whole, s);
    else if (a.x_type == RPD_DTYPE_F16)
      own_tile<F16>(q, whole, s);
    else
      own_tile<F32>(q, whole, s);
  } else {
    if (a.x_type == RPD_DTYPE_BF16)
      rows<Bf16>(q, a, s);
    else if (a.x_type == RPD_DTYPE_F16)
      rows<F16>(q, a, s);
    else
      rows<F32>(q, a, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    tile(q, whole, s);
    if (a.vt0 < a.nvt) {   // the tiles of the last round, in smaller pieces
      if ((e = hipGetLastError()) != hipSuccess) return e;
      Fp8Call last = a;
      last.tiles = a.nvt - a.vt0;
      last.nb = a.last_nb;
      last.nrt = (a.mb + a.last_nb - 1) / a.last_nb;
      tile(q, last, s);
    }
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.argmax && a.splits > 1) {
    k_fp8_join_stats<<<a.M, 256, 0, s>>>(q, a);
  } else if (a.argmax) {
    k_fp8_stats<<<a.M, 64, 0, s>>>(a);
  } else if (a.splits > 1) {
    const long long n = (long long)a.M * ((q.V + 3) / 4);
    k_fp8_join<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(q, a);
  }
  return hipGetLastError();
}

}  // namespace rpd
