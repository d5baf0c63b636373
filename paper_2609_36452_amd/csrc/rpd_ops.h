// Internal interface between the C ABI of the operators around the commit step
// (rpd_ops.cpp) and their gfx950 kernels (quant.hip, verify.hip, distill.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rpd.h"

namespace rpd {

// the calling thread's error text (rpd_api.cpp)
rpd_status fail(rpd_status s, const char* fmt, ...);
void clear_error();

inline size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

typedef unsigned int codes_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------- quant.hip --

struct QuantDims {
  int V, d, group;
  int ng;               // groups of a row
  int vt, nc;           // tiles of 16 vocabulary rows, chunks of 128 columns
  int ngp;              // groups of a row padded to whole chunks
  size_t scale_offset, zero_offset, bytes;   // of the packed head
};

struct QuantCall {
  const codes_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;   // NULL: 8 everywhere
  const uint16_t* x;      // [M][d], rows x_stride elements apart
  long long x_stride;
  bool x_vec;             // rows 16-byte aligned
  bool bf16;
  int M;
  bool stats;
  void* out;              // [M][V], rows out_stride elements apart
  long long out_stride;
  int out_type;           // RPD_DTYPE_*
  float logit_scale;
  codes_t* xrows;         // [16-row tile][chunk][4][64] operands; NULL: the workgroups convert x (at most 16 rows)
  int32_t* xexp;          // [rows] binary exponent taken out of a bf16 row
  float4* partials;       // [M][slots]
  int32_t* argmax;
  float* confidence;
  float* entropy;
  // plan
  int nc_wave, row_tiles; // template shape: chunks a wave, tiles of 16 rows a workgroup
  int waves, rounds;      // waves of a workgroup; passes of them over the columns
  int row_groups, slots;  // workgroups = row_groups x slots (a multiple of 8)
};

// tiles of 16 vocabulary rows between two barriers (and in flight), for nc
// chunks a wave and mt tiles of 16 rows: two buffers of their sums from 16 waves
// have to fit LDS
constexpr int quant_batch(int nc, int mt) { return mt == 1 ? 4 / nc : 2; }
inline size_t quant_lds_bytes(const QuantCall& a) {
  const int nb = quant_batch(a.nc_wave, a.row_tiles);
  return (size_t)2 * a.waves * nb * a.row_tiles * 1024 + (size_t)a.row_tiles * (nb * 4096 + 16 * 64 + 64);
}

hipError_t launch_quant_pack(const QuantDims& q, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros,
                             char* packed, hipStream_t s);
hipError_t launch_quant_project(const QuantDims& q, const QuantCall& a, hipStream_t s);

// ------------------------------------------------------------ verify.hip --

// a part of a row of logits: its maximum, and the sum of e^(scale (z - m)) or the maximum's lowest index
struct RowPart {
  double S;
  float m;
  int idx;
};

// the rows that a sequence draws its further token from
struct VerifyPick {
  double sp, sq;          // sums of the target's row n and, if token n was turned down, of the draft's
  float mp, mq;           // their maxima
  int x;                  // the token turned down, or -1
  int down;
};

struct VerifyCall {
  int B, T, V, dtype;
  const void* target;     // [B][T+1][V]
  long long t_batch, t_row;
  const void* draft;      // [B][T][V] or NULL
  long long d_batch, d_row;
  const int32_t* token;   // [B][T]
  const int32_t* len;     // [B] or NULL
  const float* u;         // [B][T]
  const float* r;         // [B]
  float target_scale, draft_scale;
  bool greedy;
  int32_t* out_token;     // [B][T+1]
  int32_t* n_accept;      // [B]
  float* accept;          // [B][T]
  // workspace
  RowPart* stats;         // [rows][splits]
  VerifyPick* picks;      // [B]
  double* sums;           // [2][B][parts]: of p, of max(0, p - q)
  double* totals;         // [2][B][parts]: of the exponentials of the sampled rows; NULL: the statistics are float64
  int splits, chunk;      // parts of a row, of `chunk` entries, for the statistics
  int parts, part;        // and for the sums of a sampled row
};

hipError_t launch_verify(const VerifyCall& a, hipStream_t s);

// ----------------------------------------------------------- distill.hip --

struct DistillCall {
  int N, V, k, dtype, teacher_dtype;
  const void* logits;     // [N][V]
  long long stride;
  const int32_t* ids;     // [N][k]
  const void* teacher;    // [N][k]
  const float* lse;       // [N] or NULL
  const float* weight;    // [N] or NULL
  const float* up;        // [N] or NULL
  float scale;
  float* loss;            // [N]
  float* state;           // [N][RPD_DISTILL_STATE]
  void* grad;             // [N][V] or NULL
  long long grad_stride;
  float2* partials;       // [N][splits]
  int splits, chunk;      // parts of a row, of `chunk` entries
};

hipError_t launch_distill_loss(const DistillCall& a, hipStream_t s);   // with a.grad the gradient as well
hipError_t launch_distill_grad(const DistillCall& a, hipStream_t s);

}  // namespace rpd
