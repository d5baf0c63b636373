// Output head with 4-bit weights and group scales over few rows.
//
//   y[m][v] = sum_g s[v][g] sum_{k in g} (q[v][k] - z[v][g]) x[m][k]
//
// Bound: one stream of the packed codes from HBM (half a byte a weight). What
// has to keep up with it is turning codes into matrix operands and feeding x.
// 4096 columns, V = 126464 (267 MB): 44 us for one row (6.1 TB/s); 54-59 for 32
// rows, where converting the codes and the products take as long as the stream
// (the vector instructions hold a SIMD for 56% of the time, the matrix cores for
// 24%); 96-100 for 64 rows, which convert them twice (61% and 28%). Rows of more
// than 8192 columns leave that bound: x no longer fits the registers, is loaded
// and converted anew for every tile, and the converting forms spill a few of
// them: 65536 rows of 16384 bf16 take 187 us for one row (2.9 TB/s of codes), 311
// for 16, 280 for 32; of 8192 50, 58 and 77.
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
// multiply-add instead, which saves their shift: 9 instructions for 8 weights,
// masking and setting the exponent being one.
// bf16 rows become fp16 by a power of two per row (the largest finite |x| comes
// to 2^14..2^15): their 8 bits fit, and an element so small that it falls among
// fp16's subnormals is off by at most 2^-39 of the row's largest, far below
// what fp32 accumulation keeps. fp16 rows stay as they are: among subnormal
// elements every product with q - z is a whole multiple of 2^-24, and nothing of
// it is lost (rows of 2^-22 to 2^-14 give the logits of the same rows times 2^10
// bit by bit). Sums are fp32: within a group on the matrix cores, then scaled,
// then over groups, then over waves, in a fixed order that is the same for every
// vocabulary row (equal rows give equal logits).
#include <climits>
#include <cstdint>

#include "reduce_device.h"
#include "rpd_ops.h"

namespace rpd {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
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

// Scales and zero points of tile t, chunk c: [16 rows][groups of a chunk], so that a chunk's are one or two lines
// (row by row they were 16 lines a load).
__global__ __launch_bounds__(256) void k_quant_pack_scales(QuantDims q, const uint16_t* __restrict__ scales,
                                                           const uint8_t* __restrict__ zeros,
                                                           uint16_t* __restrict__ s_out, uint8_t* __restrict__ z_out) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long n = (long long)q.vt * kTileV * q.ngp;
  if (i >= n) return;
  const int gpc = kChunk / q.group;
  const long long tc = i / (kTileV * gpc);
  const int c = (int)(tc % q.nc), in_chunk = (int)(i - tc * (kTileV * gpc));
  const long long v = tc / q.nc * kTileV + in_chunk / gpc;
  const int g = c * gpc + in_chunk % gpc;
  const bool in = v < q.V && g < q.ng;
  s_out[i] = in ? scales[v * q.ng + g] : (uint16_t)0;
  if (z_out) z_out[i] = in ? zeros[v * q.ng + g] & 15 : (uint8_t)0;
}

// ---------------------------------------------------------------- project --

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

constexpr int kRsrcFlags = 0x00020000;
constexpr int kNonTemporal = 2;   // a load's policy bits

// N bytes at a lane's offset from a uniform base; 0 beyond the range
template <int N>
__device__ __forceinline__ typename Raw<N>::t load_bits(char* base, int range, uint32_t offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, range, kRsrcFlags);
  if constexpr (N == 1)
    return __builtin_amdgcn_raw_buffer_load_b8(r, offset, 0, 0);
  else if constexpr (N == 2)
    return __builtin_amdgcn_raw_buffer_load_b16(r, offset, 0, 0);
  else if constexpr (N == 4)
    return __builtin_amdgcn_raw_buffer_load_b32(r, offset, 0, 0);
  else
    return __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, 0));
}

// 8 codes as q - z in fp16, exactly; zl and zh hold -(1024 + z) and -(64 + z).
// A nibble in the low mantissa bits of 1024 is 1024 + q, four bits up
// 1024 + 16 q: one mask-and-or each, one subtraction or multiply-add for a
// pair, one shift for the other two pairs. masks: 0x000f000f and 0x00f000f0,
// one: 1024 in both halves, in registers (as literals they do not fit into one
// instruction: 107.6 us instead of 96.2 at 64 rows). As subnormals, q 2^-24,
// the codes would need no subtraction, 5 instructions, and the zero points a
// correction by the sums of x; but the matrix cores keep fewer bits of such
// products (one instruction over normally distributed x: off by 1.3e-6 of the
// terms instead of 3e-8): logits were off by 4e-6 of their size, 1e-7 so, for 4%
// of the time at 64 rows.
__device__ __forceinline__ f16x8 decode(uint32_t w, f16x2 zl, f16x2 zh, uint32_t mask_low, uint32_t mask_high,
                                        uint32_t one) {
  const f16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  const uint32_t w8 = w >> 8;
  const uint32_t u0 = (w & mask_low) | one, u1 = (w & mask_high) | one;
  const uint32_t u2 = (w8 & mask_low) | one, u3 = (w8 & mask_high) | one;
  const f16x2 a = __builtin_bit_cast(f16x2, u0) + zl;
  const f16x2 b = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, u1), sixteenth, zh);
  const f16x2 c = __builtin_bit_cast(f16x2, u2) + zl;
  const f16x2 e = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, u3), sixteenth, zh);
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
}

template <bool BF16>
__device__ __forceinline__ float from_bits16(uint32_t b) {
  return BF16 ? __uint_as_float(b << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)b);
}

// 8 bf16 elements of a row as fp16 operands, scaled by 2^-ex
__device__ __forceinline__ u32x4 to_operand(const u32x4 r, int ex) {
  u32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t two = r[e];
    const f16x2 w = {(_Float16)ldexpf(__uint_as_float(two << 16), -ex),
                     (_Float16)ldexpf(__uint_as_float(two & 0xffff0000u), -ex)};
    o[e] = __builtin_bit_cast(uint32_t, w);
  }
  return o;
}

// One logit into a running softmax state, with one exponential: of the
// distance to the larger of z and m. NaN never becomes m and leaves S and T NaN.
__device__ __forceinline__ void soft_push(Soft& s, float z, int v) {
  const bool up = z > s.m;
  const float d = up ? s.m - z : z - s.m;       // <= 0, or NaN
  const float e = __expf(d);
  const float S0 = up ? s.S : 1.f, T0 = up ? s.T : 0.f;   // what is carried over to the new maximum
  const float dt = S0 == 0.f ? 0.f : d;         // nothing seen yet: d is -inf
  const float Sc = S0 * e, Tc = fmaf(dt, S0, T0) * e;
  s.S = Sc + (up ? 1.f : s.S);
  s.T = Tc + (up ? 0.f : s.T);
  s.idx = up ? v : s.idx;
  s.m = up ? z : s.m;
}

// NC chunks a wave, MT tiles of 16 rows, GPC groups a chunk, ZP: zero points,
// LONG: rows longer than the waves hold, x loaded anew in every round, PRE: x laid out by k_quant_rows (else the
// workgroup converts it), BF16: of that type, else fp16
template <int NC, int MT, int GPC, bool ZP, bool LONG, bool PRE, bool BF16>
__global__ __launch_bounds__(kMaxWaves * 64) void k_quant_project(QuantDims q, QuantCall a) {
  constexpr int NB = quant_batch(NC, MT);       // tiles between two barriers; as many are in flight
  typedef typename Raw<2 * GPC>::t sraw_t;
  typedef typename Raw<GPC>::t zraw_t;
  extern __shared__ __align__(16) float lds[];
  const int W = a.waves, tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nthreads = W * 64;
  // [2][W][NB][MT][64 lanes][4] partial sums, [NB][MT*256] states, [W][MT*16] maxima, [MT*16] exponents
  constexpr int kRedWave = NB * MT * 256;
  const int red_buf = W * kRedWave;
  float* red = lds;
  float4* states = reinterpret_cast<float4*>(lds + 2 * red_buf);
  uint32_t* s_max = reinterpret_cast<uint32_t*>(lds + 2 * red_buf + 4 * NB * MT * 256);
  int* s_exp = reinterpret_cast<int*>(s_max + kMaxWaves * MT * 16);
  // workgroup -> (row group, slot): the row groups of one slot run on one XCD, where they share the codes in its L2
  const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
  const int rg = local % a.row_groups, slot = local / a.row_groups * 8 + xcd;
  const int m0 = rg * MT * 16, M = min(a.M - m0, MT * 16);
  const int col = lane & 15, quad = lane >> 4;
  const int n_tiles = q.vt > slot ? (q.vt - slot + a.slots - 1) / a.slots : 0;
  const int per_round = W * NC;

  // step = (tile of this slot, round over the columns); tiles slot, slot + slots, ...
  u32x4 wb[NB][NC];
  sraw_t sb[NB][NC];
  zraw_t zb[NB][NC];
  const uint32_t w_lane = lane * 16, z_lane = col * GPC;
  constexpr int s_range = kTileV * GPC * 2;
  // The step to be fetched next. Fetches are never skipped (the last tile is fetched again instead): with one that
  // may be, the compiler cannot count the loads in flight and waits for all of them.
  const int last_tile = n_tiles > 0 ? slot + (n_tiles - 1) * a.slots : 0;
  int f_tile = min(slot, last_tile), f_round = 0;
  auto fetch = [&](int c, u32x4& w, sraw_t& s, zraw_t& z) {
    // chunks beyond the columns: the last one, whose scales are then not used
    const int chunk = min((LONG ? f_round * per_round : 0) + wid * NC + c, q.nc - 1);
    // buffer loads: a resource at the chunk and a lane's fixed offset, no 64-bit address a lane
    char* w_base = const_cast<char*>(reinterpret_cast<const char*>(a.codes)) + ((long long)f_tile * q.nc + chunk) * 1024;
    const long long entry = ((long long)f_tile * q.nc + chunk) * (kTileV * GPC);
    char* s_base = const_cast<char*>(reinterpret_cast<const char*>(a.scales)) + entry * 2;
    char* z_base = const_cast<char*>(reinterpret_cast<const char*>(a.zeros)) + entry;
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(w_base, (short)0, 1024, kRsrcFlags);
    w = __builtin_amdgcn_raw_buffer_load_b128(wr, w_lane, 0, kNonTemporal);
    s = load_bits<2 * GPC>(s_base, s_range, 2 * z_lane);
    if (ZP) z = load_bits<GPC>(z_base, s_range / 2, z_lane);
  };
  auto fetched = [&]() {
    if (!LONG || ++f_round == a.rounds) {
      f_round = 0;
      f_tile = min(f_tile + a.slots, last_tile);
    }
  };
#pragma unroll
  for (int u = 0; u < NB; ++u) {
#pragma unroll
    for (int c = 0; c < NC; ++c) fetch(c, wb[u][c], sb[u][c], zb[u][c]);
    fetched();
  }

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
  u32x4 xf[MT][NC][4];   // as loaded, then the fp16 operands
  auto load_x = [&](int round) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int chunk = round * per_round + wid * NC + c;
          if (!PRE) {
            xf[mt][c][u] = x_piece(mt, chunk, u);
          } else {
            xf[mt][c][u] = u32x4{0u, 0u, 0u, 0u};
            if (chunk < q.nc) xf[mt][c][u] = a.xrows[((long long)(rg * MT + mt) * q.nc + chunk) * 256 + u * 64 + lane];
          }
        }
  };
  if (!BF16) {
    if (tid < MT * 16) s_exp[tid] = 0;
    if (!PRE && !LONG) load_x(0);
  } else if (PRE) {
    if (tid < MT * 16) s_exp[tid] = a.xexp[rg * MT * 16 + tid];
  } else {
    // each row's largest magnitude (the bits of magnitudes are in order; infinity and NaN count as the largest finite
    // one, the row's logits being infinite or NaN anyway)
    const u16x2 finite = {(uint16_t)0x7f7f, (uint16_t)0x7f7f};
    u16x2 big[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) big[mt] = u16x2{0, 0};
    for (int round = 0; round < (LONG ? a.rounds : 1); ++round) {
      load_x(round);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              big[mt] = __builtin_elementwise_max(big[mt], __builtin_bit_cast(u16x2, xf[mt][c][u][e] & 0x7fff7fffu));
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      big[mt] = __builtin_elementwise_min(big[mt], finite);
      uint32_t m = max((uint32_t)big[mt].x, (uint32_t)big[mt].y);
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      if (quad == 0) s_max[wid * MT * 16 + mt * 16 + col] = m;
    }
    __syncthreads();
    if (tid < MT * 16) {
      uint32_t b = 0;
      for (int w = 0; w < W; ++w) b = max(b, s_max[w * MT * 16 + tid]);
      int e = 15;
      if (b) (void)frexpf(__uint_as_float(b << 16), &e);   // in [2^(e-1), 2^e): to be brought to 2^14..2^15
      s_exp[tid] = e - 15;
    }
  }
  if (a.stats)
    for (int e = tid; e < NB * MT * 256; e += nthreads) states[e] = soft_pack(soft_empty());
  __syncthreads();

  auto convert_x = [&]() {
    if (PRE || !BF16) return;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int ex = s_exp[mt * 16 + col];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          u32x4 o = to_operand(xf[mt][c][u], ex);
          asm volatile("" : "+v"(o));   // packed here: one piece at a time in float beside the rows
          xf[mt][c][u] = o;
        }
    }
  };
  if (PRE && !LONG) load_x(0);
  if (!LONG) convert_x();

  auto row_of = [&](int e) { return 16 * (e >> 8) + 4 * (e >> 6 & 3) + (e >> 4 & 3); };
  // not literals, see decode
  uint32_t mask = 0x000f000fu, one = 0x64006400u;
  asm("" : "+s"(mask), "+v"(one));
  int buf = 0;
  for (int ti = 0; ti < n_tiles; ti += NB) {
    // a batch of tiles, over the end the last one again (its sums are then not used)
    float* dst = red + buf * red_buf + wid * kRedWave + lane * 4;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      f32x4 acc[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int round = 0; round < (LONG ? a.rounds : 1); ++round) {
        if (LONG) {
          load_x(round);
          convert_x();
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
          for (int g = 0; g < GPC; ++g) {
            const uint32_t bits = (uint32_t)(sb[u][c] >> (16 * g)) & 0xffffu;
            const float sc = from_bits16<BF16>((LONG ? round * per_round : 0) + wid * NC + c < q.nc ? bits : 0u);
            const _Float16 z = ZP ? (_Float16)(float)(uint32_t)(zb[u][c] >> (8 * g) & 255) : (_Float16)8.f;
            const _Float16 zl1 = (_Float16)-1024.f - z, zh1 = (_Float16)-64.f - z;
            const f16x2 zl = {zl1, zl1}, zh = {zh1, zh1};
            f32x4 part[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) part[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = g * 4 / GPC; t < (g + 1) * 4 / GPC; ++t) {
              const f16x8 wf = decode(wb[u][c][t], zl, zh, mask, mask << 4, one);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
                part[mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, xf[mt][c][t]), wf, part[mt],
                                                                  0, 0, 0);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[mt][i] = fmaf(sc, part[mt][i], acc[mt][i]);
            if (GPC > 1 && NC * MT > 2) {
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+v"(acc[mt]));
            }
          }
          fetch(c, wb[u][c], sb[u][c], zb[u][c]);   // into the registers just read
        }
        fetched();
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (16 * mt + 4 * quad < M) *reinterpret_cast<f32x4*>(dst + (u * MT + mt) * 256) = acc[mt];
    }
    // the batch's sums over the waves, out to memory or into the states. The next batch's partial sums go to the
    // other buffer, so one barrier a batch is enough.
    lds_barrier();
    const float* src = red + buf * red_buf;
    buf ^= 1;
    for (int i = tid; i < NB * MT * 256; i += nthreads) {
      // entry of a tile: v fastest, 16 columns, then the 4 rows of a quad (a wave reads 64 consecutive words), then
      // quad and tile of rows
      const int b = i / (MT * 256), e = i - b * (MT * 256);
      const int m = row_of(e);
      const long long v = (slot + (long long)(ti + b) * a.slots) * kTileV + (e & 15);
      if (m >= M || v >= q.V) continue;
      const float* p = src + b * MT * 256 + (e >> 8) * 256 + ((e >> 6 & 3) * 16 + (e & 15)) * 4 + (e >> 4 & 3);
      float z = 0.f;
      int w = 0;
      for (; w + 8 <= W; w += 8, p += 8 * kRedWave) {
        float t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = p[k * kRedWave];
#pragma unroll
        for (int k = 0; k < 8; ++k) z += t[k];
      }
      for (; w < W; ++w, p += kRedWave) z += *p;
      z = ldexpf(z, s_exp[m]);
      if (a.stats) {   // this thread has entry i in every batch
        Soft st = soft_unpack(states[i]);
        soft_push(st, z * a.logit_scale, (int)v);
        states[i] = soft_pack(st);
        continue;
      }
      const long long at = (m0 + m) * a.out_stride + v;
      if (a.out_type == 1)
        static_cast<float*>(a.out)[at] = z;
      else if (a.out_type == 0)
        static_cast<__bf16*>(a.out)[at] = (__bf16)z;
      else
        static_cast<_Float16*>(a.out)[at] = (_Float16)z;
    }
  }
  if (!a.stats) return;
  // a row's states, of the batch's tiles and then of 16 columns, in a fixed order
  __syncthreads();
  for (int e = tid; e < MT * 256; e += nthreads) {
    Soft st = soft_unpack(states[e]);
#pragma unroll
    for (int b = 1; b < NB; ++b) st = soft_merge(st, soft_unpack(states[b * MT * 256 + e]));
#pragma unroll
    for (int k = 1; k < 16; k <<= 1) st = soft_merge(st, soft_shfl_xor(st, k));
    if ((e & 15) == 0 && row_of(e) < M) a.partials[(long long)(m0 + row_of(e)) * a.slots + slot] = soft_pack(st);
  }
}

// Rows of x as fp16 operands in the order in which k_quant_project reads them,
// one workgroup a row (rows past the last as zeros): for more than 16 rows,
// where every workgroup converting all of them for itself cost it 12 us (32
// rows of 4096: the loads, 64 bytes a row, crowd the caches, and 2.6 us of
// conversion).
template <bool BF16>
__global__ __launch_bounds__(256) void k_quant_rows(QuantDims q, QuantCall a) {
  const int m = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  __shared__ uint32_t s_max[4];
  const uint16_t* x = a.x + m * a.x_stride;
  auto piece = [&](int k) {
    u32x4 r = {0u, 0u, 0u, 0u};
    if (m >= a.M || k >= q.d) return r;
    if (a.x_vec) return *reinterpret_cast<const u32x4*>(x + k);
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (uint32_t)x[k + 2 * e] | (uint32_t)x[k + 2 * e + 1] << 16;
    return r;
  };
  const int pieces = q.nc * 16, rt = m >> 4, col = m & 15;
  constexpr int kHeld = 4;   // a thread's first pieces are read once (rows of up to 8192)
  u32x4 held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) held[j] = piece(8 * (tid + 256 * j));
  int ex = 0;
  if (BF16) {
    u16x2 big = {0, 0};
    auto grow = [&](const u32x4 r) {
#pragma unroll
      for (int e = 0; e < 4; ++e) big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2, r[e] & 0x7fff7fffu));
    };
#pragma unroll
    for (int j = 0; j < kHeld; ++j) grow(held[j]);
    for (int p = tid + 256 * kHeld; p < pieces; p += 256) grow(piece(8 * p));
    uint32_t top = min((uint32_t)max(big.x, big.y), 0x7f7fu);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, k));
    if (lane == 0) s_max[tid >> 6] = top;
    __syncthreads();
    top = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    int e = 15;
    if (top) (void)frexpf(__uint_as_float(top << 16), &e);
    ex = e - 15;
    if (tid == 0) a.xexp[m] = ex;
  }
  auto put = [&](int p, const u32x4 r) {
    if (p < pieces)
      a.xrows[((long long)rt * q.nc + (p >> 4)) * 256 + (p >> 2 & 3) * 64 + (p & 3) * 16 + col] =
          BF16 ? to_operand(r, ex) : r;
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j) put(tid + 256 * j, held[j]);
  for (int p = tid + 256 * kHeld; p < pieces; p += 256) put(p, piece(8 * p));
}

// one wave a row: the slots' states -> argmax, top probability, entropy
__global__ __launch_bounds__(64) void k_quant_stats(QuantCall a) {
  const int m = blockIdx.x, lane = threadIdx.x;
  float4 keep[8];
  const Soft st = wave_merge_row(a.partials + (long long)m * a.slots, a.slots, lane, keep);
  if (lane == 0) {
    a.argmax[m] = st.idx == INT_MAX ? -1 : st.idx;   // a row of NaN has none
    a.confidence[m] = 1.f / st.S;
    a.entropy[m] = logf(st.S) - st.T / st.S;
  }
}

template <int NC, int MT, int GPC, bool LONG, bool PRE>
hipError_t project_z(const QuantDims& q, const QuantCall& a, hipStream_t s) {
  const size_t lds = quant_lds_bytes(a);
  auto kernel = a.zeros ? (a.bf16 ? k_quant_project<NC, MT, GPC, true, LONG, PRE, true>
                                  : k_quant_project<NC, MT, GPC, true, LONG, PRE, false>)
                        : (a.bf16 ? k_quant_project<NC, MT, GPC, false, LONG, PRE, true>
                                  : k_quant_project<NC, MT, GPC, false, LONG, PRE, false>);
  if (lds > 64 * 1024) {   // what a launch may have without asking
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<a.slots * a.row_groups, a.waves * 64, lds, s>>>(q, a);
  return hipGetLastError();
}

template <int NC, int MT, bool PRE, bool LONG = false>
hipError_t project_g(const QuantDims& q, const QuantCall& a, hipStream_t s) {
  switch (q.group) {
    case 32: return project_z<NC, MT, 4, LONG, PRE>(q, a, s);
    case 64: return project_z<NC, MT, 2, LONG, PRE>(q, a, s);
    default: return project_z<NC, MT, 1, LONG, PRE>(q, a, s);
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
  const bool pre = a.xrows != nullptr;
  if (pre) {
    const int rows = a.row_groups * a.row_tiles * 16;
    if (a.bf16)
      k_quant_rows<true><<<rows, 256, 0, s>>>(q, a);
    else
      k_quant_rows<false><<<rows, 256, 0, s>>>(q, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.nc_wave == 1)
    e = pre ? project_g<1, 2, true>(q, a, s) : project_g<1, 1, false>(q, a, s);
  else if (a.nc_wave == 2)
    e = pre ? project_g<2, 2, true>(q, a, s) : project_g<2, 1, false>(q, a, s);
  else if (a.rounds == 1)
    e = pre ? project_g<4, 1, true>(q, a, s) : project_g<4, 1, false>(q, a, s);
  else
    e = pre ? project_g<4, 1, true, true>(q, a, s) : project_g<4, 1, false, true>(q, a, s);
  if (e != hipSuccess || !a.stats) return e;
  k_quant_stats<<<a.M, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace rpd
