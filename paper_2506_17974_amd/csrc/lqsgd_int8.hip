// gfx950 kernels of the linear layer on 8-bit rows.
//
// Sums of products are exact 32-bit integers: the same whatever their order.
#include "lqsgd_block_kernels.h"
#include "lqsgd_linear_device.h"

#include <algorithm>
#include <cstdint>

namespace lqsgd {
namespace linear {
namespace {

// v_mfma_i32_32x32x32_i8: a lane holds 16 consecutive r of operand row (lane mod 32), r0 = 16 (lane / 32); D comes back with
// i = 8 (v / 4) + 4 (lane / 32) + v mod 4 in register v, j = lane mod 32.
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;

// The end of a product: v holds the sums of D[j][i0 .. i0 + N - 1].
template <typename T, int N>
__device__ inline void finish(const int (&sum)[N], const Int8Args& a, int64_t j, int i0) {
  const int n = j < a.nj ? a.ni - i0 : 0;
  if (n <= 0) return;
  const float sb = a.scales_b[j];
  float v[N], scale[N], bias[N] = {};
  load_values(scale, a.scales_a + i0, n);
  if (a.bias) load_values(bias, static_cast<const T*>(a.bias) + i0, n);
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = fmaf((float)sum[k], sb * scale[k], bias[k]);
  activate_all(v, a.act);
  if (a.residual) {
    float r[N];
    load_values(r, static_cast<const T*>(a.residual) + j * a.ldr + i0, n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += r[k];
  }
  store_values(static_cast<T*>(a.out) + j * a.ldo + i0, v, n);
}

// A tile of 64 x 64 to a workgroup of four wavefronts, 32 x 32 each, operands from memory as the matrix instructions take them.
template <typename T>
__global__ __launch_bounds__(256) void int8_product_kernel(Int8Args a, int tiles_i) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = (int)(blockIdx.x % tiles_i) * 64 + (wave & 1) * 32;
  const int64_t j0 = (int64_t)(blockIdx.x / tiles_i) * 64 + (wave >> 1) * 32;
  const int8_t* pa = a.a + (int64_t)min(i0 + (lane & 31), a.ni - 1) * a.stride + 16 * (lane >> 5);
  const int8_t* pb = a.b + min(j0 + (lane & 31), a.nj - 1) * a.stride + 16 * (lane >> 5);
  i32x16 acc = {};
  for (int r = 0; r < a.stride; r += 32)
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4*>(pa + r), *reinterpret_cast<const i32x4*>(pb + r), acc, 0, 0, 0);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int sum[4] = {acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
    finish<T>(sum, a, j0 + (lane & 31), i0 + 8 * g + 4 * (lane >> 5));
  }
}

}  // namespace

hipError_t launch_int8_product(int type, const Int8Args& a, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    const int tiles_i = (a.ni + 63) / 64;
    const int64_t tiles = tiles_i * ((a.nj + 63) / 64);
    if (tiles * 256 >= int64_t(1) << 32) return hipErrorInvalidValue;
    int8_product_kernel<T><<<dim3((unsigned)tiles), 256, 0, s>>>(a, tiles_i);
    return hipGetLastError();
  });
}

}  // namespace linear
}  // namespace lqsgd
