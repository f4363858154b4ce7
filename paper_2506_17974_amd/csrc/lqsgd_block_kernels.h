// Argument blocks and launchers of the gfx950 kernels around the linear layer: norm, 8-bit rows, dropout, the product of 8-bit rows.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lqsgd_linear_kernels.h"

namespace lqsgd {
namespace linear {

struct Rows {                                     // 8-bit rows' memory; codes == nullptr: none
  int8_t* codes;
  float* scales;
};

struct NormArgs {
  int64_t samples;
  int32_t features;
  double eps, inverse;                            // inverse: 1 / features, the launcher's
  const void* x; int64_t ldx;
  const void* residual; int64_t ldr;              // the rest may be nullptr
  const void* gain;
  void* h; int64_t ldh;
  void* y; int64_t ldy;
  float* rstd;
  Codes kept;
  Rows rows;
};

struct NormBackwardArgs {
  int64_t samples;
  int32_t features;
  const void* dy; int64_t lddy;
  const void* h; int64_t ldh;                     // nullptr: held
  Codes held;
  const float* rstd;
  const void* gain;                               // may be nullptr, like all below
  const void* dh; int64_t lddh;
  void* dx; int64_t lddx;
  float* dgain;
  int32_t accumulate;
  void* workspace;
  int* arrived;                                   // as in ProductArgs; the kernel: nullptr where another joins the runs' sums
};

struct DropoutArgs {
  int64_t samples;
  int32_t features;
  uint32_t least;                                 // 0 .. 65536: bits from which a value stays
  float factor;
  uint64_t seed, offset;
  const uint64_t* more_offset;                    // may be nullptr, like residual and kept
  const void* x; int64_t ldx;
  const void* residual; int64_t ldr;
  void* y; int64_t ldy;
  Codes kept;
};

struct Int8Args {                                 // D[j][i] = sum over r of A[i][r] B[j][r]: A the weight, B the input
  int64_t nj;
  int32_t ni, stride;                             // stride: of the codes' rows, a multiple of 32; zeros behind the depth
  const int8_t* a; const float* scales_a;
  const int8_t* b; const float* scales_b;
  const void* bias; const void* residual; int64_t ldr;
  void* out; int64_t ldo;
  int32_t act;
  void* workspace;
  int* arrived;
};

hipError_t launch_rows_save(int type, int64_t samples, int32_t features, const void* x, int64_t ldx, Rows rows, hipStream_t s);
hipError_t launch_rows_load(int type, int64_t samples, int32_t features, Rows rows, void* x, int64_t ldx, hipStream_t s);
hipError_t launch_rms_norm(int type, const NormArgs& a, hipStream_t s);
hipError_t launch_rms_norm_backward(int type, const NormBackwardArgs& a, hipStream_t s);
hipError_t launch_dropout(int type, const DropoutArgs& a, hipStream_t s);
hipError_t launch_int8_product(int type, const Int8Args& a, hipStream_t s);

}  // namespace linear
}  // namespace lqsgd
