// gfx950 kernels of the linear layer whose gradients the compressor takes: the three products of a layer (forward with its
// epilogue, input gradient, weight gradient from an 8-bit checkpoint), checkpoints, and the activation's backward pass.
//
// Sums have a fixed order: results are bit-identical run to run.
#include "lqsgd_linear_kernels.h"

#include <algorithm>
#include <cstdint>
#include <type_traits>

namespace lqsgd {
namespace linear {
namespace {

// ---------------------------------------------------------------------------
// types, checkpoints, activations
// ---------------------------------------------------------------------------
using bf16 = __bf16;
using f16 = _Float16;

__device__ inline float widen(float v) { return v; }
__device__ inline float widen(bf16 v) { return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16); }
__device__ inline float widen(f16 v) { return (float)v; }
template <typename T> __device__ inline T narrow(float v) { return (T)v; }      // to nearest even

// Bounds of a checkpoint's e: every q 2^e, |q| <= 127, is a number of the type.
template <typename T> struct Exponents { static constexpr int lo = -126, hi = 121; };
template <> struct Exponents<f16> { static constexpr int lo = -24, hi = 9; };

__device__ inline uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
__device__ inline float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// e of a group from the largest magnitude's bits (as integers magnitudes are ordered, infinities and NaN last).  absmax =
// m 2^E, 1 <= m < 2, takes e = E - 6, or E - 5 from 127.5 2^(E-6) on: adding 2^-7 of the mantissa carries into the exponent there.
template <typename T>
__device__ inline int group_exponent(uint32_t absmax) {
  const int e = (int)((absmax + 0x10000u) >> 23) - 133;
  return min(max(e, Exponents<T>::lo), Exponents<T>::hi);
}
__device__ inline bool group_finite(uint32_t absmax) { return absmax < 0x7f800000u; }
__device__ inline uint32_t code_of(float v, float inverse_step) {
  return (uint32_t)(int)fminf(fmaxf(rintf(v * inverse_step), -127.f), 127.f) & 0xffu;
}
// What a code's factor is: 2^e, NaN for byte 255.
__device__ inline float factor_of(uint32_t byte) {
  return byte == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
}

// Phi(z) = erfc(-z / sqrt 2) / 2 by the rational form of Hastings (Abramowitz and Stegun 7.1.26, |error| <= 1.5e-7): with
// t = 1 / (1 + p |x|), erfc(|x|) = (a1 t + ... + a5 t^5) exp(-x^2).  Half the instructions of a correctly rounded erf, and its
// error is that of a few fp32 operations.  `density`: exp(-z^2 / 2).
__device__ inline float normal_cdf(float z, float* density) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
  const float g = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * g;
  *density = g;
  return z > 0.f ? 1.f - tail : tail;
}
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }

__device__ inline float activate(float z, int act) {
  float d;
  switch (act) {
    case kRelu: return z < 0.f ? 0.f : z;           // keeps NaN
    case kGelu: return z * normal_cdf(z, &d);
    case kSilu: return z * sigmoid(z);
    default: return z;
  }
}
__device__ inline float slope(float z, int act) {
  switch (act) {
    case kRelu: return z > 0.f ? 1.f : z == z ? 0.f : z;
    case kGelu: {
      float g;
      const float c = normal_cdf(z, &g);
      return fmaf(0.39894228040143268f * z, g, c);
    }
    case kSilu: {
      const float s = sigmoid(z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// N consecutive values from memory of any alignment, `n` of them there; the others read as 0.
template <int N, typename T>
__device__ inline void load_values(float (&v)[N], const T* p, int n) {
  if (n >= N) {
    T t[N];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = widen(t[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < n ? widen(p[k]) : 0.f;
  }
}
template <int N, typename T>
__device__ inline void store_values(T* p, const float (&v)[N], int n) {
  if (n >= N) {
    T t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = narrow<T>(v[k]);
    __builtin_memcpy(p, t, sizeof t);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < n) p[k] = narrow<T>(v[k]);
  }
}

// N values of one group quantised and packed, four to a word; `absmax` is the whole group's.
template <typename T, int N>
__device__ inline void pack_codes(uint32_t (&w)[N / 4], const float (&v)[N], uint32_t absmax, uint32_t* byte) {
  const bool finite = group_finite(absmax);
  const int e = group_exponent<T>(absmax);
  const float inv = power_of_two(-e);
#pragma unroll
  for (int k = 0; k < N / 4; ++k)
    w[k] = code_of(v[4 * k], inv) | code_of(v[4 * k + 1], inv) << 8 | code_of(v[4 * k + 2], inv) << 16 | code_of(v[4 * k + 3], inv) << 24;
  if (!finite) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) w[k] = 0u;
  }
  *byte = finite ? (uint32_t)(e + 127) : 255u;
}

// ---------------------------------------------------------------------------
// checkpoints
// ---------------------------------------------------------------------------
// A thread takes 8 consecutive values, four lanes a group; a workgroup a run of 256 such pieces of the whole tensor, rows end to
// end, so that narrow tensors fill their lanes too.  Bound by memory: s + 33/32 bytes per value.
constexpr int kPiece = 8;

template <typename T>
__global__ __launch_bounds__(256) void checkpoint_save_kernel(const T* x, int64_t ldx, Codes c, int64_t samples, int features, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x;
  const int64_t row = row0 + at / pieces;
  const uint32_t piece = at % pieces;
  const bool there = row < samples;
  float v[kPiece];
  load_values(v, x + row * ldx + piece * kPiece, there ? features - (int)(piece * kPiece) : 0);
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < kPiece; ++k) m = max(m, magnitude_bits(v[k]));
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  m = max(m, (uint32_t)__shfl_xor((int)m, 2));
  uint32_t w[2], byte;
  pack_codes<T>(w, v, m, &byte);
  if (!there) return;
  *reinterpret_cast<uint2*>(c.codes + row * ((int64_t)pieces * kPiece) + piece * kPiece) = make_uint2(w[0], w[1]);
  if ((piece & 3u) == 0) c.exponents[row * (pieces >> 2) + (piece >> 2)] = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(256) void checkpoint_load_kernel(T* x, int64_t ldx, Codes c, int64_t samples, int features, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x;
  const int64_t row = row0 + at / pieces;
  const uint32_t piece = at % pieces;
  if (row >= samples) return;
  const uint2 w = *reinterpret_cast<const uint2*>(c.codes + row * ((int64_t)pieces * kPiece) + piece * kPiece);
  const float f = factor_of(c.exponents[row * (pieces >> 2) + (piece >> 2)]);
  float v[kPiece];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k] = (float)(int8_t)(w.x >> (8 * k)) * f;
    v[4 + k] = (float)(int8_t)(w.y >> (8 * k)) * f;
  }
  store_values(x + row * ldx + piece * kPiece, v, features - (int)(piece * kPiece));
}

// ---------------------------------------------------------------------------
// activation backward
// ---------------------------------------------------------------------------
// A workgroup takes a strip of 8 << lanes_log2 features and a run of samples; a lane keeps 8 features' sums.  Lanes that the strip
// does not fill take further samples.  Strips' sums over runs go to `part` (runs x rows) where there is more than one run.
template <typename T>
__global__ __launch_bounds__(256) void activation_backward_kernel(const T* dy, int64_t lddy, Codes z, T* dz, int64_t lddz, float* dbias,
                                                                  int accumulate, float* part, int64_t samples, int rows, int act,
                                                                  int lanes_log2, int64_t run) {
  __shared__ float sums[256][kPiece + 1];
  const int lanes = 1 << lanes_log2, t = threadIdx.x;
  const int feature = ((int)blockIdx.x * lanes + (t & (lanes - 1))) * kPiece;
  const int n = rows - feature;
  const int groups = (rows + kGroup - 1) / kGroup;
  const int64_t first = (int64_t)blockIdx.y * run, last = min(samples, first + run);
  float s[kPiece] = {};
  if (n > 0) {
    for (int64_t m = first + (t >> lanes_log2); m < last; m += 256 >> lanes_log2) {
      float v[kPiece];
      load_values(v, dy + m * lddy + feature, n);
      if (act != kNone) {
        const uint2 w = *reinterpret_cast<const uint2*>(z.codes + m * ((int64_t)groups * kGroup) + feature);
        const float f = factor_of(z.exponents[m * groups + feature / kGroup]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] *= slope((float)(int8_t)(w.x >> (8 * k)) * f, act);
          v[4 + k] *= slope((float)(int8_t)(w.y >> (8 * k)) * f, act);
        }
      }
      if (dz) store_values(dz + m * lddz + feature, v, n);
#pragma unroll
      for (int k = 0; k < kPiece; ++k) s[k] += v[k];
    }
  }
  if (!dbias) return;
#pragma unroll
  for (int k = 0; k < kPiece; ++k) sums[t][k] = s[k];
  __syncthreads();
  // a thread adds up one feature over the samples' lanes
  const int wide = lanes * kPiece;
  for (int i = t; i < wide; i += 256) {
    const int f = (int)blockIdx.x * wide + i;
    if (f >= rows) break;
    float total = 0.f;
    for (int k = i / kPiece; k < 256; k += lanes) total += sums[k][i % kPiece];
    if (part) part[(int64_t)blockIdx.y * rows + f] = total;
    else dbias[f] = accumulate ? dbias[f] + total : total;
  }
}

__global__ __launch_bounds__(256) void sum_runs_kernel(const float* part, float* dbias, int accumulate, int rows, int runs) {
  __shared__ float sums[4][64];
  const int f = (int)blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float s = 0.f;
  if (f < rows)
    for (int k = w; k < runs; k += 4) s += part[(int64_t)k * rows + f];
  sums[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && f < rows) {
    s = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    dbias[f] = accumulate ? dbias[f] + s : s;
  }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
// The end of a product: v holds D[j][i0 .. i0 + 15], the lane `partner` away the other half of the group of 32 (i0 a multiple of
// 16).  All lanes of the wavefront come here together; `there` is false for those that have no row j.
template <typename T, int PRODUCT>
__device__ inline void finish(float (&v)[16], const ProductArgs& a, int64_t j, int i0, bool there, int partner) {
  const int n = there ? a.ni - i0 : 0;
  if (PRODUCT == kWeightGrad) {
    if (n <= 0) return;
    if (a.out_type == kF32) {
      float* out = static_cast<float*>(a.out) + j * a.ldo + i0;
      if (a.accumulate) {
        float before[16];
        load_values(before, out, n);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] += before[k];
      }
      store_values(out, v, n);
    } else {
      bf16* out = static_cast<bf16*>(a.out) + j * a.ldo + i0;
      if (a.accumulate) {
        float before[16];
        load_values(before, out, n);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] += before[k];
      }
      store_values(out, v, n);
    }
    return;
  }
  T* out = static_cast<T*>(a.out) + j * a.ldo + i0;
  if (PRODUCT == kInputGrad) {
    if (n > 0) store_values(out, v, n);
    return;
  }
  const int groups = (a.ni + kGroup - 1) / kGroup;
  const bool in_codes = there && i0 < groups * kGroup;
  const int64_t code_at = j * ((int64_t)groups * kGroup) + i0, exp_at = j * groups + i0 / kGroup;
  if (a.bias) {
    float b[16];
    load_values(b, static_cast<const T*>(a.bias) + i0, n);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] += b[k];
  }
  auto keep = [&](const Codes& c) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k >= n) v[k] = 0.f;
      m = max(m, magnitude_bits(v[k]));
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, partner));
    uint32_t w[4], byte;
    pack_codes<T>(w, v, m, &byte);
    if (in_codes) {
      *reinterpret_cast<uint4*>(c.codes + code_at) = make_uint4(w[0], w[1], w[2], w[3]);
      if ((i0 & 16) == 0) c.exponents[exp_at] = (uint8_t)byte;
    }
  };
  if (a.z.codes) keep(a.z);
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = activate(v[k], a.act);
  if (a.residual) {
    float r[16];
    load_values(r, static_cast<const T*>(a.residual) + j * a.ldr + i0, n);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] += r[k];
  }
  if (n > 0) store_values(out, v, n);
  if (a.y.codes) {
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = widen(narrow<T>(v[k]));
    keep(a.y);
  }
}

// One operand value, 0 outside.
template <typename T, int PRODUCT>
__device__ inline float operand_a(const ProductArgs& a, int i, int64_t r) {
  if (i >= a.ni || r >= a.depth) return 0.f;
  if (PRODUCT == kForward) return widen(static_cast<const T*>(a.a)[i * a.lda + r]);
  if (PRODUCT == kInputGrad) return widen(static_cast<const T*>(a.a)[r * a.lda + i]);
  const int groups = (a.ni + kGroup - 1) / kGroup;
  const float f = factor_of(a.held.exponents[r * groups + i / kGroup]);
  return widen(narrow<T>((float)a.held.codes[r * ((int64_t)groups * kGroup) + i] * f));
}
template <typename T, int PRODUCT>
__device__ inline float operand_b(const ProductArgs& a, int64_t j, int64_t r) {
  if (j >= a.nj || r >= a.depth) return 0.f;
  return widen(static_cast<const T*>(a.b)[PRODUCT == kWeightGrad ? r * a.ldb + j : j * a.ldb + r]);
}

// 64 x 64 of D to a workgroup, 16 a thread, operands through LDS 16 deep.
template <typename T, int PRODUCT>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs a, int tiles_i) {
  __shared__ float ta[16][68], tb[16][68];
  const int i0 = (int)(blockIdx.x % tiles_i) * 64;
  const int64_t j0 = (int64_t)(blockIdx.x / tiles_i) * 64;
  const int t = threadIdx.x, j = t >> 2, ii = (t & 3) * 16;
  float v[16] = {};
  for (int64_t r0 = 0; r0 < a.depth; r0 += 16) {
    for (int k = t; k < 1024; k += 256) {
      const int i = PRODUCT == kForward ? k >> 4 : k & 63, ra = PRODUCT == kForward ? k & 15 : k >> 6;
      ta[ra][i] = operand_a<T, PRODUCT>(a, i0 + i, r0 + ra);
      const int jj = PRODUCT == kWeightGrad ? k & 63 : k >> 4, rb = PRODUCT == kWeightGrad ? k >> 6 : k & 15;
      tb[rb][jj] = operand_b<T, PRODUCT>(a, j0 + jj, r0 + rb);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float b = tb[r][j];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = fmaf(ta[r][ii + k], b, v[k]);
    }
    __syncthreads();
  }
  finish<T, PRODUCT>(v, a, j0 + j, i0 + ii, j0 + j < a.nj, 1);
}

template <typename T, int PRODUCT>
hipError_t product(const ProductArgs& a, hipStream_t s) {
  const int64_t tiles_i = (a.ni + 63) / 64, tiles_j = (a.nj + 63) / 64;
  if (tiles_i * tiles_j > INT32_MAX) return hipErrorInvalidValue;
  product_kernel<T, PRODUCT><<<dim3((unsigned)(tiles_i * tiles_j)), 256, 0, s>>>(a, (int)tiles_i);
  return hipGetLastError();
}

template <typename F>
hipError_t by_type(int type, F&& f) {
  switch (type) {
    case kF32: return f(float{});
    case kBF16: return f(bf16{});
    case kF16: return f(f16{});
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_product(int product_kind, int type, const ProductArgs& a, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    switch (product_kind) {
      case kForward: return product<T, kForward>(a, s);
      case kInputGrad: return product<T, kInputGrad>(a, s);
      default: return product<T, kWeightGrad>(a, s);
    }
  });
}

hipError_t launch_checkpoint_save(int type, int64_t samples, int32_t features, const void* x, int64_t ldx, Codes c, hipStream_t s) {
  const uint32_t pieces = (uint32_t)((features + kGroup - 1) / kGroup * (kGroup / kPiece));
  const int64_t blocks = (samples * pieces + 255) / 256;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    checkpoint_save_kernel<T><<<dim3((unsigned)blocks), 256, 0, s>>>(static_cast<const T*>(x), ldx, c, samples, features, pieces);
    return hipGetLastError();
  });
}

hipError_t launch_checkpoint_load(int type, int64_t samples, int32_t features, Codes c, void* x, int64_t ldx, hipStream_t s) {
  const uint32_t pieces = (uint32_t)((features + kGroup - 1) / kGroup * (kGroup / kPiece));
  const int64_t blocks = (samples * pieces + 255) / 256;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    checkpoint_load_kernel<T><<<dim3((unsigned)blocks), 256, 0, s>>>(static_cast<T*>(x), ldx, c, samples, features, pieces);
    return hipGetLastError();
  });
}

hipError_t launch_activation_backward(int type, int act, int64_t samples, int32_t rows, const void* dy, int64_t lddy, Codes z, void* dz,
                                      int64_t lddz, float* dbias, int accumulate, void* workspace, hipStream_t s) {
  const int pieces = (rows + kPiece - 1) / kPiece;
  int lanes_log2 = 0;
  while ((1 << lanes_log2) < pieces && lanes_log2 < 6) ++lanes_log2;
  const int strips = (pieces + (1 << lanes_log2) - 1) >> lanes_log2;
  const int64_t at_once = 256 >> lanes_log2;
  const int64_t most = std::max<int64_t>(1, 2048 / strips);
  const int64_t rounds = std::max<int64_t>(4, (samples + at_once * most - 1) / (at_once * most));
  const int64_t run = rounds * at_once;
  const int64_t runs = std::max<int64_t>(1, (samples + run - 1) / run);
  float* part = dbias && runs > 1 ? static_cast<float*>(workspace) : nullptr;
  hipError_t e = by_type(type, [&](auto zero) {
    using T = decltype(zero);
    activation_backward_kernel<T><<<dim3((unsigned)strips, (unsigned)runs), 256, 0, s>>>(
        static_cast<const T*>(dy), lddy, z, static_cast<T*>(dz), lddz, dbias, accumulate, part, samples, rows, act, lanes_log2, run);
    return hipGetLastError();
  });
  if (e != hipSuccess || !part) return e;
  sum_runs_kernel<<<dim3((unsigned)((rows + 63) / 64)), 256, 0, s>>>(part, dbias, accumulate, rows, (int)runs);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace lqsgd
