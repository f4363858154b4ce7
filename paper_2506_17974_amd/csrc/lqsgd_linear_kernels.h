// Argument blocks and launchers of the linear layer's gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "lqsgd_linear_plan.h"

namespace lqsgd {
namespace linear {

constexpr int kGroup = 32;                        // features that share an exponent in a checkpoint
constexpr int kSlopeRows = 40;                    // exponents whose codes' slopes are not all 1/2, or 0 and 1
constexpr int kSlopeFloats = 2 * kSlopeRows * 128;       // slopes of gelu and silu for every code of those

enum Type { kF32 = 0, kBF16 = 1, kF16 = 2 };
enum Act { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };

struct Codes {                                    // a checkpoint's memory; codes == nullptr: none
  int8_t* codes;
  uint8_t* exponents;
};

struct ProductArgs {                              // sizes as in lqsgd_linear_plan.h
  int64_t nj, depth;
  int32_t ni;
  const void* a; int64_t lda;                     // kWeightGrad: unused, the operand is `held`
  const void* b; int64_t ldb;
  Codes held;
  const void* bias; const void* residual; int64_t ldr;     // kForward
  Codes z, y;                                     // kForward
  void* out; int64_t ldo;
  int32_t act;
  int32_t out_type;                               // kWeightGrad: kF32 or kBF16
  int32_t accumulate;                             // kWeightGrad
  void* workspace;
  int* arrived;                                   // kTiles zeros: parts of a tile's sum that have come; the kernels leave zeros
};

hipError_t launch_product(int product, int type, const ProductArgs& a, hipStream_t s);
hipError_t launch_checkpoint_save(int type, int64_t samples, int32_t features, const void* x, int64_t ldx, Codes c, hipStream_t s);
hipError_t launch_checkpoint_load(int type, int64_t samples, int32_t features, Codes c, void* x, int64_t ldx, hipStream_t s);
hipError_t launch_activation_backward(int type, int act, int64_t samples, int32_t rows, const void* dy, int64_t lddy, Codes z, void* dz,
                                      int64_t lddz, float* dbias, int accumulate, void* workspace, const float* slopes, hipStream_t s);
hipError_t launch_prepare(float* slopes, int* arrived, hipStream_t s);       // kSlopeFloats and kTiles of them, once for a context

}  // namespace linear
}  // namespace lqsgd
