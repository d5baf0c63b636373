// Output head with 4-bit weights and group scales over few rows.
//
//   y[m][v] = sum_g s[v][g] sum_{k in g} (q[v][k] - z[v][g]) x[m][k]
//
// Bound: one stream of the packed codes from HBM (half a byte a weight). What
// has to keep up with it is turning codes into matrix operands and feeding x.
//
// x stays: the waves of a workgroup divide the columns among them, each keeps
// the fp16 fragments of its columns of all rows in registers, and only the
// codes stream past, in tiles of 16 vocabulary rows. (x read from LDS for every
// tile would move four times the bytes of the codes at 16 rows.) A tile's sums
// over the waves' columns meet in LDS.
//
// The matrix operands are exact: a code nibble put into the mantissa of fp16
// 1024 is 1024 + q, and one packed subtraction leaves q - z, an integer in
// -15..15. Bits 4..7 of each half are 1024 + 16 q and take one packed
// multiply-add instead, which saves their shift: 9 instructions for 8 weights.
// bf16 rows become fp16 by a power of two per row (the largest finite |x| comes
// to 2^14..2^15): their 8 bits fit, and an element so small that it falls among
// fp16's subnormals is off by at most 2^-40 of the row's largest, far below
// what fp32 accumulation keeps. Sums are fp32: within a group on the matrix
// cores, then scaled, then over groups, then over waves, in a fixed order that
// is the same for every vocabulary row (equal rows give equal logits).
#include <cstdint>

#include "rpd_device.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;

constexpr int kTileV = 16;     // vocabulary rows of a tile
constexpr int kChunk = 128;    // columns of a chunk: 16 bytes of codes a lane
constexpr int kMaxWaves = 16;

// ------------------------------------------------------------------- pack --
//
// Tile t, chunk c: 64 lanes x 16 bytes; lane l holds row 16 t + l % 16, its
// dword u the columns 128 c + 32 u + 8 (l / 16) + 0..7, the order in which the
// matrix cores take them. Inside a dword column 2 i sits at nibble i, column
// 2 i + 1 at nibble i + 4, so that one mask takes a pair. Rows and columns
// beyond the head hold code 0 and scale 0.
__global__ __launch_bounds__(256) void k_quant_pack(QuantDims q, const uint8_t* __restrict__ codes,
                                                    uint32_t* __restrict__ out) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long n = (long long)q.vt * q.nc * 64;
  if (i >= n) return;
  const int lane = (int)(i & 63);
  const long long tc = i >> 6;
  const int c = (int)(tc % q.nc);
  const long long v = tc / q.nc * kTileV + (lane & 15);
  uint32_t w[4] = {0, 0, 0, 0};
  if (v < q.V) {
    const uint8_t* row = codes + v * (q.d / 2);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int k = kChunk * c + 32 * u + 8 * (lane >> 4);
      if (k >= q.d) continue;   // d is a multiple of 8
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint32_t two = row[k / 2 + b];
        w[u] |= (two & 15u) << (4 * b) | (two >> 4) << (4 * b + 16);
      }
    }
  }
  u32x4 o = {w[0], w[1], w[2], w[3]};
  reinterpret_cast<u32x4*>(out)[i] = o;
}

// scales and zero points: [16 vt][ngp], rows padded to whole chunks
__global__ __launch_bounds__(256) void k_quant_pack_scales(QuantDims q, const uint16_t* __restrict__ scales,
                                                           const uint8_t* __restrict__ zeros,
                                                           uint16_t* __restrict__ s_out, uint8_t* __restrict__ z_out) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long n = (long long)q.vt * kTileV * q.ngp;
  if (i >= n) return;
  const long long v = i / q.ngp;
  const int g = (int)(i - v * q.ngp);
  const bool in = v < q.V && g < q.ng;
  s_out[i] = in ? scales[v * q.ng + g] : (uint16_t)0;
  if (z_out) z_out[i] = in ? zeros[v * q.ng + g] & 15 : (uint8_t)0;
}

// ---------------------------------------------------------------- project --

__device__ __forceinline__ f16x2 as_h2(uint32_t u) { return __builtin_bit_cast(f16x2, u); }

// 8 codes -> q - z in fp16; zl = -(1024 + z), zh = -(64 + z) in both halves
__device__ __forceinline__ f16x8 decode(uint32_t w, f16x2 zl, f16x2 zh) {
  const f16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  const uint32_t w8 = w >> 8;
  const f16x2 a = as_h2((w & 0x000f000fu) | 0x64006400u) + zl;
  const f16x2 b = __builtin_elementwise_fma(as_h2((w & 0x00f000f0u) | 0x64006400u), sixteenth, zh);
  const f16x2 c = as_h2((w8 & 0x000f000fu) | 0x64006400u) + zl;
  const f16x2 e = __builtin_elementwise_fma(as_h2((w8 & 0x00f000f0u) | 0x64006400u), sixteenth, zh);
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
}

template <int N>
struct Raw;
template <>
struct Raw<1> { typedef uint8_t t; };
template <>
struct Raw<2> { typedef uint16_t t; };
template <>
struct Raw<4> { typedef uint32_t t; };
template <>
struct Raw<8> { typedef uint64_t t; };

__device__ __forceinline__ float from_bits16(uint32_t b, bool bf16) {
  return bf16 ? __uint_as_float(b << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)b);
}

// one logit into a running softmax state (an entry that is NaN leaves S and T NaN)
__device__ __forceinline__ void soft_push(Soft& s, float z, int v) {
  const bool up = z > s.m;
  const float M = up ? z : s.m;
  const float dm = s.S == 0.f ? 0.f : s.m - M, dz = z - M;
  const float em = __expf(dm), ez = __expf(dz);
  s.T = (s.T + dm * s.S) * em + ez * dz;
  s.S = s.S * em + ez;
  s.idx = up ? v : s.idx;
  s.m = M;
}

// NC chunks a wave, MT tiles of 16 rows, GPC groups a chunk, ZP: zero points
template <int NC, int MT, int GPC, bool ZP>
__global__ __launch_bounds__(kMaxWaves * 64) void k_quant_project(QuantDims q, QuantCall a) {
  constexpr int D = 2;   // tiles of codes in flight
  typedef typename Raw<2 * GPC>::t sraw_t;
  typedef typename Raw<GPC>::t zraw_t;
  extern __shared__ __align__(16) float lds[];
  const int W = a.waves, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int nthreads = W * 64;
  // [2][W][NB][MT][64 lanes][4] partial sums, [MT*256] states, [W][MT*16] maxima, [MT*16] exponents
  const int red_wave = a.nb * MT * 256, red_buf = W * red_wave;
  float* red = lds;
  float4* states = reinterpret_cast<float4*>(lds + 2 * red_buf);
  float* s_max = lds + 2 * red_buf + 4 * MT * 256;
  int* s_exp = reinterpret_cast<int*>(s_max + kMaxWaves * MT * 16);
  // workgroup -> (row group, slot): the row groups of one slot run on one XCD, where they share the codes in its L2
  const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
  const int rg = local % a.row_groups, slot = local / a.row_groups * 8 + xcd;
  const int m0 = rg * MT * 16, M = min(a.M - m0, MT * 16);
  const int col = lane & 15, quad = lane >> 4;
  const bool bf16 = a.bf16;

  auto x_piece = [&](int mt, int chunk, int u) {   // 8 elements of row 16 mt + col, 0 beyond the rows and columns
    const int m = 16 * mt + col, k = kChunk * chunk + 32 * u + 8 * quad;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (m < M && k < q.d) {
      const uint16_t* p = a.x + (m0 + m) * a.x_stride + k;
      if (a.x_vec) {
        r = *reinterpret_cast<const u32x4*>(p);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (uint32_t)p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
      }
    }
    return r;
  };
  const int per_round = W * NC;
  if (bf16) {
    // the exponent that brings each row's largest finite element to 2^14..2^15
    uint32_t big[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) big[mt] = 0;
    for (int c = wid; c < q.nc; c += W)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const u32x4 r = x_piece(mt, c, u);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t lo = r[e] & 0x7fffu, hi = r[e] >> 16 & 0x7fffu;
            big[mt] = max(big[mt], max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
          }
        }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      big[mt] = max(big[mt], (uint32_t)__shfl_xor((int)big[mt], 16));
      big[mt] = max(big[mt], (uint32_t)__shfl_xor((int)big[mt], 32));
      if (quad == 0) s_max[wid * MT * 16 + mt * 16 + col] = __uint_as_float(big[mt] << 16);
    }
    __syncthreads();
    if (tid < MT * 16) {
      float b = 0.f;
      for (int w = 0; w < W; ++w) b = fmaxf(b, s_max[w * MT * 16 + tid]);
      int e = 0;
      if (b > 0.f) (void)frexpf(b, &e);   // b in [2^(e-1), 2^e)
      s_exp[tid] = b > 0.f ? e - 15 : 0;
    }
  } else if (tid < MT * 16) {
    s_exp[tid] = 0;
  }
  for (int e = tid; e < MT * 256; e += nthreads) states[e] = soft_pack(soft_empty());
  __syncthreads();

  f16x8 xf[MT][NC][4];
  auto load_x = [&](int round) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int ex = s_exp[mt * 16 + col];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int chunk = round * per_round + wid * NC + c;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const u32x4 r = x_piece(mt, chunk, u);
          if (bf16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              xf[mt][c][u][2 * e] = (_Float16)ldexpf(__uint_as_float(r[e] << 16), -ex);
              xf[mt][c][u][2 * e + 1] = (_Float16)ldexpf(__uint_as_float(r[e] & 0xffff0000u), -ex);
            }
          } else {
            xf[mt][c][u] = __builtin_bit_cast(f16x8, r);
          }
        }
      }
    }
  };
  if (a.rounds == 1) load_x(0);

  // step = (tile of this slot, round over the columns); tiles slot, slot + slots, ...
  const int n_tiles = q.vt > slot ? (q.vt - slot + a.slots - 1) / a.slots : 0;
  const int steps = n_tiles * a.rounds;
  u32x4 wb[D][NC];
  sraw_t sb[D][NC];
  zraw_t zb[D][NC];
  auto fetch = [&](int step, u32x4(&w)[NC], sraw_t(&s)[NC], zraw_t(&z)[NC]) {
    const int ti = step / a.rounds, round = step - ti * a.rounds;
    const long long tile = slot + (long long)ti * a.slots;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int chunk = round * per_round + wid * NC + c;
      const bool in = chunk < q.nc;
      const int cc = in ? chunk : 0;   // a wave beyond the columns reads chunk 0 and multiplies it by x = 0
      w[c] = a.codes[(tile * q.nc + cc) * 64 + lane];
      s[c] = reinterpret_cast<const sraw_t*>(a.scales)[(tile * kTileV + col) * q.nc + cc];
      if (ZP) z[c] = reinterpret_cast<const zraw_t*>(a.zeros)[(tile * kTileV + col) * q.nc + cc];
    }
  };
#pragma unroll
  for (int u = 0; u < D; ++u)
    if (u < steps) fetch(u, wb[u], sb[u], zb[u]);

  int nb = 0, buf = 0, first_tile = 0;
  f32x4 acc[MT];
  // the sums of the last nb tiles over the waves, out to memory or into the states
  auto finish = [&](int count) {
    lds_barrier();
    const float* src = red + buf * red_buf;
    for (int e = tid; e < MT * 256; e += nthreads) {
      // v fastest: 16 columns, then the 4 rows of a quad (64 consecutive words a wave), then quad and tile of rows
      const int c16 = e & 15, i = e >> 4 & 3, qd = e >> 6 & 3, mt = e >> 8;
      const int m = 16 * mt + 4 * qd + i;
      if (m >= M) continue;
      const int word = mt * 256 + (qd * 16 + c16) * 4 + i, ex = s_exp[m];
      Soft st;
      if (a.stats) st = soft_unpack(states[e]);
      for (int b = 0; b < count; ++b) {
        float z = 0.f;
        for (int w = 0; w < W; ++w) z += src[w * red_wave + b * MT * 256 + word];
        z = ldexpf(z, ex);
        const long long v = (slot + (long long)(first_tile + b) * a.slots) * kTileV + c16;
        if (v >= q.V) continue;
        if (a.stats) {
          soft_push(st, z * a.logit_scale, (int)v);
        } else {
          const long long at = (m0 + m) * a.out_stride + v;
          if (a.out_type == 1)
            static_cast<float*>(a.out)[at] = z;
          else if (a.out_type == 0)
            static_cast<__bf16*>(a.out)[at] = (__bf16)z;
          else
            static_cast<_Float16*>(a.out)[at] = (_Float16)z;
        }
      }
      if (a.stats) states[e] = soft_pack(st);
    }
    buf ^= 1;
    nb = 0;
  };

  for (int s0 = 0; s0 < steps; s0 += D) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      const int step = s0 + u;
      if (step >= steps) break;
      const int ti = step / a.rounds, round = step - ti * a.rounds;
      if (a.rounds > 1) load_x(round);
      if (round == 0) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int g = 0; g < GPC; ++g) {
          _Float16 zf = (_Float16)8.f;
          if (ZP) zf = (_Float16)(float)(uint32_t)(zb[u][c] >> (8 * g) & 255);
          const _Float16 zl1 = (_Float16)-1024.f - zf, zh1 = (_Float16)-64.f - zf;
          const f16x2 zl = {zl1, zl1}, zh = {zh1, zh1};
          f32x4 part[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) part[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = g * 4 / GPC; t < (g + 1) * 4 / GPC; ++t) {
            const f16x8 wf = decode(wb[u][c][t], zl, zh);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              part[mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[mt][c][t], wf, part[mt], 0, 0, 0);
          }
          const float sc = from_bits16((uint32_t)(sb[u][c] >> (16 * g) & 0xffff), bf16);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[mt][i] = fmaf(sc, part[mt][i], acc[mt][i]);
        }
      }
      if (step + D < steps) fetch(step + D, wb[u], sb[u], zb[u]);
      if (round + 1 < a.rounds) continue;
      if (nb == 0) first_tile = ti;
      float* dst = red + buf * red_buf + wid * red_wave + nb * MT * 256;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (16 * mt + 4 * quad < M) *reinterpret_cast<f32x4*>(dst + mt * 256 + lane * 4) = acc[mt];
      if (++nb == a.nb || ti + 1 == n_tiles) finish(nb);
    }
  }
  if (!a.stats) return;
  // the 16 columns' states of each row, in a fixed order
  __syncthreads();
  for (int m = tid; m < M; m += nthreads) {
    Soft st = soft_empty();
    for (int c16 = 0; c16 < 16; ++c16)
      st = soft_merge(st, soft_unpack(states[(m >> 4) * 256 + (m >> 2 & 3) * 64 + (m & 3) * 16 + c16]));
    a.partials[(long long)(m0 + m) * a.slots + slot] = soft_pack(st);
  }
}

// one wave a row: the slots' states -> argmax, top probability, entropy
__global__ __launch_bounds__(64) void k_quant_stats(QuantCall a) {
  const int m = blockIdx.x, lane = threadIdx.x;
  Soft st = soft_empty();
  for (int i = lane; i < a.slots; i += 64) st = soft_merge(st, soft_unpack(a.partials[(long long)m * a.slots + i]));
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) st = soft_merge(st, soft_shfl_xor(st, k));
  if (lane == 0) {
    a.argmax[m] = st.idx;
    a.confidence[m] = 1.f / st.S;
    a.entropy[m] = logf(st.S) - st.T / st.S;
  }
}

template <int NC, int MT, int GPC>
hipError_t project_z(const QuantDims& q, const QuantCall& a, hipStream_t s) {
  const size_t lds = quant_lds_bytes(a);
  auto kernel = a.zeros ? k_quant_project<NC, MT, GPC, true> : k_quant_project<NC, MT, GPC, false>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)lds);
  if (e != hipSuccess) return e;
  kernel<<<a.slots * a.row_groups, a.waves * 64, lds, s>>>(q, a);
  return hipGetLastError();
}

template <int NC, int MT>
hipError_t project_g(const QuantDims& q, const QuantCall& a, hipStream_t s) {
  switch (q.group) {
    case 32: return project_z<NC, MT, 4>(q, a, s);
    case 64: return project_z<NC, MT, 2>(q, a, s);
    default: return project_z<NC, MT, 1>(q, a, s);
  }
}

}  // namespace

hipError_t launch_quant_pack(const QuantDims& q, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros,
                             char* packed, hipStream_t s) {
  const long long n = (long long)q.vt * q.nc * 64, ns = (long long)q.vt * kTileV * q.ngp;
  k_quant_pack<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(q, codes, reinterpret_cast<uint32_t*>(packed));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_quant_pack_scales<<<(unsigned)((ns + 255) / 256), 256, 0, s>>>(
      q, scales, zeros, reinterpret_cast<uint16_t*>(packed + q.scale_offset),
      zeros ? reinterpret_cast<uint8_t*>(packed + q.zero_offset) : nullptr);
  return hipGetLastError();
}

hipError_t launch_quant_project(const QuantDims& q, const QuantCall& a, hipStream_t s) {
  hipError_t e;
  if (a.nc_wave == 1)
    e = a.row_tiles == 1 ? project_g<1, 1>(q, a, s) : project_g<1, 2>(q, a, s);
  else if (a.nc_wave == 2)
    e = a.row_tiles == 1 ? project_g<2, 1>(q, a, s) : project_g<2, 2>(q, a, s);
  else
    e = project_g<4, 1>(q, a, s);
  if (e != hipSuccess || !a.stats) return e;
  k_quant_stats<<<a.M, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace rpd
