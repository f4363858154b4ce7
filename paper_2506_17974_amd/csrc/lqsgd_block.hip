// gfx950 kernels of what stands around the linear layer: the root-mean-square norm and its backward pass, 8-bit rows, dropout.
//
// Sums have a fixed order: results are bit-identical run to run.
#include "lqsgd_block_kernels.h"
#include "lqsgd_linear_device.h"

#include <algorithm>
#include <cstdint>

namespace lqsgd {
namespace linear {
namespace {

// ---------------------------------------------------------------------------
// a row shared out among lanes
// ---------------------------------------------------------------------------
// 8-bit rows: the step of a row whose largest magnitude is absmax (NaN if that is none).
__device__ inline float row_step(float absmax) {
  return absmax < __builtin_inff() ? fmaxf(absmax / 127.f, 0x1p-126f) : __builtin_nanf("");
}
// Codes of 8 values, `inverse` = 1 / step; 0 where that is NaN.  |v| inverse is 127 (1 + 2^-22) at most, which rounds to 127; the product is
// rounded before the sum that rounds it to an integer, as the definition has it.
__device__ inline uint2 row_codes(const float (&v)[kPiece], float inverse) {
#pragma clang fp contract(off)
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t q[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) q[c] = __builtin_bit_cast(uint32_t, v[4 * k + c] * inverse + 12582912.f);
    const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
    w[k] = inverse == inverse ? low | high : 0u;
  }
  return make_uint2(w[0], w[1]);
}

// ---------------------------------------------------------------------------
// norm and 8-bit rows
// ---------------------------------------------------------------------------
// THREADS to a row, PIECES of 8 values each in registers; WIDE: a row of any length, read again for its outputs.  ROWS rows to a
// workgroup (of a wavefront each).  NORM: the norm, with what is wanted of it; otherwise 8-bit rows of x alone.
template <typename T, int THREADS, int PIECES, int ROWS, bool NORM, bool WIDE>
__global__ __launch_bounds__(THREADS * ROWS) void row_kernel(NormArgs a) {
  static_assert(ROWS == 1 || THREADS == 64, "rows that share a workgroup have a wavefront each");
  constexpr int kWaves = THREADS / 64;
  const int t = threadIdx.x % THREADS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  if (ROWS > 1 && row >= a.samples) return;
  const int n = a.features, stride = (n + kGroup - 1) / kGroup * kGroup;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const r = NORM && a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  const T* const gain = NORM ? static_cast<const T*>(a.gain) : nullptr;
  T* const h = NORM && a.h ? static_cast<T*>(a.h) + row * a.ldh : nullptr;

  // values of the row from `col` on, as the norm sees them; zeros behind its end
  auto load = [&](float (&v)[kPiece], int col) {
    load_values(v, x + col, n - col);
    if (r) {
      float more[kPiece];
      load_values(more, r + col, n - col);
#pragma unroll
      for (int k = 0; k < kPiece; ++k) v[k] = widen(narrow<T>(v[k] + more[k]));
    }
  };
  auto load_gain = [&](float (&g)[kPiece], int col) {
    if (gain) {
      load_values(g, gain + col, n - col);
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) g[k] = 1.f;
    }
  };
  double sum = 0.0;
  float most = 0.f;
  auto count = [&](const float (&v)[kPiece], int col) {
    if (NORM) {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) sum = __builtin_fma((double)v[k], (double)v[k], sum);
    }
    if (!NORM) {
      most = __builtin_elementwise_maximum(most, largest(v));
    } else if (a.rows.codes) {
      float g[kPiece];
      load_gain(g, col);
#pragma unroll
      for (int k = 0; k < kPiece; ++k) g[k] *= v[k];
      most = __builtin_elementwise_maximum(most, largest(g));
    }
  };

  float v[PIECES][kPiece];
  const int pieces = (n + kPiece - 1) / kPiece;
  if constexpr (WIDE) {
    for (int p = t; p < pieces; p += THREADS) {
      load(v[0], p * kPiece);
      if (h) store_values(h + p * kPiece, v[0], n - p * kPiece);
      count(v[0], p * kPiece);
    }
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) load(v[p], (t + p * THREADS) * kPiece);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * THREADS) * kPiece;
      if (h) store_values(h + col, v[p], n - col);
      count(v[p], col);
    }
  }
  if (NORM) sum = over_wave(sum, Plus{});
  if (!NORM || a.rows.codes) most = over_wave(most, Larger{});
  if constexpr (kWaves > 1) {
    __shared__ double sums[kWaves];
    __shared__ float mosts[kWaves];
    if ((t & 63) == 0) sums[t >> 6] = sum, mosts[t >> 6] = most;
    __syncthreads();
    sum = 0.0, most = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) sum += sums[k], most = __builtin_elementwise_maximum(most, mosts[k]);
  }
  const float rstd = NORM ? (float)(1.0 / sqrt(sum / n + a.eps)) : 1.f;
  const float step = row_step(most), inverse = 1.f / step;
  if (t == 0) {
    if (NORM && a.rstd) a.rstd[row] = rstd;
    if (a.rows.codes) a.rows.scales[row] = NORM ? step * rstd : step;
  }
  auto write = [&](const float (&v)[kPiece], int col) {
    float g[kPiece];
    if (NORM) {
      load_gain(g, col);
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) g[k] = 1.f;
    }
    if (a.rows.codes) {
      float q[kPiece];
#pragma unroll
      for (int k = 0; k < kPiece; ++k) q[k] = NORM ? v[k] * g[k] : v[k];
      const uint2 w = row_codes(q, inverse);
      if (col < stride) *reinterpret_cast<uint2*>(a.rows.codes + row * stride + col) = w;
    }
    if (!NORM || (!a.y && !a.kept.codes)) return;
#pragma unroll
    for (int k = 0; k < kPiece; ++k) g[k] *= v[k] * rstd;
    if (a.y) store_values(static_cast<T*>(a.y) + row * a.ldy + col, g, n - col);
    if (!a.kept.codes) return;
#pragma unroll
    for (int k = 0; k < kPiece; ++k) g[k] = widen(narrow<T>(g[k]));
    uint32_t w[2], byte;
    pack_codes<T>(w, g, group_largest<kPiece>(largest(g)), &byte);
    if (col >= stride) return;
    *reinterpret_cast<uint2*>(a.kept.codes + row * stride + col) = make_uint2(w[0], w[1]);
    if (col % kGroup == 0) a.kept.exponents[row * (stride / kGroup) + col / kGroup] = (uint8_t)byte;
  };
  if constexpr (WIDE) {
    // whole wavefronts go round together: lanes exchange what a group's largest value is
    for (int p = t; p < (pieces + 63) / 64 * 64; p += THREADS) {
      const int col = p * kPiece;
      if (h) {
        load_values(v[0], h + col, n - col);      // this thread's own; x or the residual may be gone
      } else {
        load(v[0], col);
      }
      write(v[0], col);
    }
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) write(v[p], (t + p * THREADS) * kPiece);
  }
}

template <typename T, bool NORM>
hipError_t run_rows(const NormArgs& all, hipStream_t s) {
  // a launch has fewer than 2^32 threads
  constexpr int64_t kSlab = int64_t(1) << 21;
  const int64_t stride = (all.features + kGroup - 1) / kGroup * kGroup;
  for (int64_t at = 0; at < all.samples; at += kSlab) {
    NormArgs a = all;
    a.samples = std::min(kSlab, all.samples - at);
    a.x = static_cast<const T*>(all.x) + at * all.ldx;
    if (a.residual) a.residual = static_cast<const T*>(all.residual) + at * all.ldr;
    if (a.h) a.h = static_cast<T*>(all.h) + at * all.ldh;
    if (a.y) a.y = static_cast<T*>(all.y) + at * all.ldy;
    if (a.rstd) a.rstd += at;
    if (a.kept.codes) a.kept = Codes{all.kept.codes + at * stride, all.kept.exponents + at * (stride / kGroup)};
    if (a.rows.codes) a.rows = Rows{all.rows.codes + at * stride, all.rows.scales + at};
    const unsigned n = (unsigned)a.samples;
    if (a.features <= 512) row_kernel<T, 64, 1, 4, NORM, false><<<dim3((n + 3) / 4), 256, 0, s>>>(a);
    else if (a.features <= 1024) row_kernel<T, 64, 2, 4, NORM, false><<<dim3((n + 3) / 4), 256, 0, s>>>(a);
    else if (a.features <= 2048) row_kernel<T, 256, 1, 1, NORM, false><<<dim3(n), 256, 0, s>>>(a);
    else if (a.features <= 4096) row_kernel<T, 256, 2, 1, NORM, false><<<dim3(n), 256, 0, s>>>(a);
    else if (a.features <= 8192) row_kernel<T, 512, 2, 1, NORM, false><<<dim3(n), 512, 0, s>>>(a);
    else if (a.features <= 16384) row_kernel<T, 512, 4, 1, NORM, false><<<dim3(n), 512, 0, s>>>(a);
    else row_kernel<T, 1024, 1, 1, NORM, true><<<dim3(n), 1024, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
__global__ __launch_bounds__(256) void rows_load_kernel(T* x, int64_t ldx, Rows rows, int64_t samples, int features, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  if (row >= samples) return;
  const uint2 w = *reinterpret_cast<const uint2*>(rows.codes + row * ((int64_t)pieces * kPiece) + piece * kPiece);
  float v[kPiece];
  decode(v, w, rows.scales[row]);
  store_values(x + row * ldx + piece * kPiece, v, features - (int)(piece * kPiece));
}

// ---------------------------------------------------------------------------
// the norm's backward pass
// ---------------------------------------------------------------------------
// What 8 values of h are, from the tensor or from its checkpoint.
template <typename T, bool HELD>
__device__ inline void load_h(float (&v)[kPiece], const NormBackwardArgs& a, int64_t row, int col) {
  const int n = a.features, groups = (n + kGroup - 1) / kGroup;
  if constexpr (HELD) {
    if (col < n) {                               // codes go on to the end of their group
      const uint2 w = *reinterpret_cast<const uint2*>(a.held.codes + row * ((int64_t)groups * kGroup) + col);
      decode(v, w, factor_of(a.held.exponents[row * groups + col / kGroup]));
#pragma unroll
      for (int k = 0; k < kPiece; ++k) v[k] = k < n - col ? v[k] : 0.f;
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) v[k] = 0.f;
    }
  } else {
    load_values(v, static_cast<const T*>(a.h) + row * a.ldh + col, n - col);
  }
}
template <typename T>
__device__ inline void load_or_ones(float (&g)[kPiece], const void* from, int col, int n) {
  if (from) {
    load_values(g, static_cast<const T*>(from) + col, n - col);
  } else {
#pragma unroll
    for (int k = 0; k < kPiece; ++k) g[k] = 1.f;
  }
}

// A workgroup takes a run of rows, ROWS at a time, THREADS to a row; a thread keeps its columns' gain and sums.  dgain: `part`, runs x
// features, where it is wanted.
template <typename T, bool HELD, int THREADS, int PIECES, int ROWS>
__global__ __launch_bounds__(THREADS * ROWS) void norm_backward_kernel(NormBackwardArgs a, float* part, int64_t run) {
  static_assert(ROWS == 1 || THREADS == 64, "rows that share a workgroup have a wavefront each");
  constexpr int kWaves = THREADS / 64;
  const int t = threadIdx.x % THREADS, slot = threadIdx.x / THREADS, n = a.features;
  const int64_t first = (int64_t)blockIdx.x * run, last = min(a.samples, first + run);
  float gain[PIECES][kPiece], sums[PIECES][kPiece] = {};
#pragma unroll
  for (int p = 0; p < PIECES; ++p) load_or_ones<T>(gain[p], a.gain, (t + p * THREADS) * kPiece, n);
  __shared__ float dots[2][kWaves];
  int turn = 0;
  for (int64_t row = first + slot; row < last; row += ROWS, turn ^= 1) {
    float dy[PIECES][kPiece], h[PIECES][kPiece];
    const float rstd = a.rstd[row];
    float dot = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * THREADS) * kPiece;
      load_values(dy[p], static_cast<const T*>(a.dy) + row * a.lddy + col, n - col);
      load_h<T, HELD>(h[p], a, row, col);
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int k = 0; k < kPiece; ++k) {
        h[p][k] *= rstd;
        sums[p][k] = fmaf(dy[p][k], h[p][k], sums[p][k]);
        dy[p][k] *= gain[p][k];
        dot = fmaf(dy[p][k], h[p][k], dot);
      }
    if (!a.dx) continue;
    dot = over_wave(dot, Plus{});
    if constexpr (kWaves > 1) {
      if ((t & 63) == 0) dots[turn][t >> 6] = dot;
      __syncthreads();
      dot = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) dot += dots[turn][k];
    }
    const float along = dot / (float)n;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * THREADS) * kPiece;
      float d[kPiece] = {};
      if (a.dh) load_values(d, static_cast<const T*>(a.dh) + row * a.lddh + col, n - col);
#pragma unroll
      for (int k = 0; k < kPiece; ++k) d[k] = fmaf(rstd, fmaf(-h[p][k], along, dy[p][k]), d[k]);
      store_values(static_cast<T*>(a.dx) + row * a.lddx + col, d, n - col);
    }
  }
  if (!part) return;
  float* const out = part + (int64_t)blockIdx.x * n;
  if constexpr (ROWS > 1) {
    __shared__ float all[ROWS][PIECES * 64 * kPiece];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int k = 0; k < kPiece; ++k) all[slot][(t + p * THREADS) * kPiece + k] = sums[p][k];
    __syncthreads();
    for (int f = threadIdx.x; f < n; f += THREADS * ROWS) {
      float total = 0.f;
#pragma unroll
      for (int k = 0; k < ROWS; ++k) total += all[k][f];
      out[f] = total;
    }
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int k = 0; k < kPiece; ++k) {
        const int f = (t + p * THREADS) * kPiece + k;
        if (f < n) out[f] = sums[p][k];
      }
  }
}

// Rows of any length, in two: each row's mean of v h rstd, then dx and the columns' sums by strips of 2048 features and runs of rows.
template <typename T, bool HELD>
__global__ __launch_bounds__(1024) void norm_along_kernel(NormBackwardArgs a, float* along) {
  __shared__ float dots[16];
  const int64_t row = blockIdx.x;
  const int n = a.features;
  const float rstd = a.rstd[row];
  float dot = 0.f;
  for (int col = (int)threadIdx.x * kPiece; col < n; col += 1024 * kPiece) {
    float dy[kPiece], h[kPiece], g[kPiece];
    load_values(dy, static_cast<const T*>(a.dy) + row * a.lddy + col, n - col);
    load_h<T, HELD>(h, a, row, col);
    load_or_ones<T>(g, a.gain, col, n);
#pragma unroll
    for (int k = 0; k < kPiece; ++k) dot = fmaf(dy[k] * g[k], h[k] * rstd, dot);
  }
  dot = over_wave(dot, Plus{});
  if ((threadIdx.x & 63) == 0) dots[threadIdx.x >> 6] = dot;
  __syncthreads();
  if (threadIdx.x != 0) return;
  dot = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) dot += dots[k];
  along[row] = dot / (float)n;
}

template <typename T, bool HELD>
__global__ __launch_bounds__(256) void norm_strips_kernel(NormBackwardArgs a, const float* along, float* part, int64_t run) {
  const int n = a.features, col = ((int)blockIdx.x * 256 + (int)threadIdx.x) * kPiece;
  if (col >= n) return;
  const int64_t first = (int64_t)blockIdx.y * run, last = min(a.samples, first + run);
  float gain[kPiece], sums[kPiece] = {};
  load_or_ones<T>(gain, a.gain, col, n);
  for (int64_t row = first; row < last; ++row) {
    float dy[kPiece], h[kPiece], d[kPiece] = {};
    const float rstd = a.rstd[row], c = along[row];
    load_values(dy, static_cast<const T*>(a.dy) + row * a.lddy + col, n - col);
    load_h<T, HELD>(h, a, row, col);
    if (a.dh) load_values(d, static_cast<const T*>(a.dh) + row * a.lddh + col, n - col);
#pragma unroll
    for (int k = 0; k < kPiece; ++k) {
      const float v = h[k] * rstd;
      sums[k] = fmaf(dy[k], v, sums[k]);
      d[k] = fmaf(rstd, fmaf(-v, c, dy[k] * gain[k]), d[k]);
    }
    if (a.dx) store_values(static_cast<T*>(a.dx) + row * a.lddx + col, d, n - col);
  }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < kPiece; ++k)
    if (col + k < n) part[(int64_t)blockIdx.y * n + col + k] = sums[k];
}

constexpr int64_t kAlong = int64_t(1) << 22;              // rows whose means lie in front of the parts in the workspace
constexpr int64_t kPartFloats = (int64_t)(kWorkspaceBytes / 4) - kAlong;

template <typename T, bool HELD>
hipError_t run_norm_backward(const NormBackwardArgs& all, hipStream_t s) {
  float* const along = static_cast<float*>(all.workspace);
  float* const parts = along + kAlong;
  const int64_t groups = (all.features + kGroup - 1) / kGroup;
  int64_t at = 0;
  do {
    NormBackwardArgs a = all;
    a.samples = std::min(kAlong, all.samples - at);
    a.accumulate = all.accumulate || at > 0;
    a.dy = static_cast<const T*>(all.dy) + at * all.lddy;
    if (a.h) a.h = static_cast<const T*>(all.h) + at * all.ldh;
    if (a.held.codes) a.held = Codes{all.held.codes + at * groups * kGroup, all.held.exponents + at * groups};
    a.rstd = all.rstd + at;
    if (a.dh) a.dh = static_cast<const T*>(all.dh) + at * all.lddh;
    if (a.dx) a.dx = static_cast<T*>(all.dx) + at * all.lddx;
    const int64_t most = std::min<int64_t>(a.features <= 16384 ? 1024 : std::max<int64_t>(1, 1024 * 2048 / a.features), kPartFloats / a.features);
    const int rows = a.features <= 1024 ? 4 : 1;
    const int64_t run = std::max<int64_t>(1, (a.samples + most * rows - 1) / (most * rows)) * rows;
    const unsigned runs = (unsigned)((a.samples + run - 1) / run);
    float* const part = a.dgain ? parts : nullptr;
    if (a.samples > 0) {
      if (a.features <= 512) norm_backward_kernel<T, HELD, 64, 1, 4><<<dim3(runs), 256, 0, s>>>(a, part, run);
      else if (a.features <= 1024) norm_backward_kernel<T, HELD, 64, 2, 4><<<dim3(runs), 256, 0, s>>>(a, part, run);
      else if (a.features <= 2048) norm_backward_kernel<T, HELD, 256, 1, 1><<<dim3(runs), 256, 0, s>>>(a, part, run);
      else if (a.features <= 4096) norm_backward_kernel<T, HELD, 256, 2, 1><<<dim3(runs), 256, 0, s>>>(a, part, run);
      else if (a.features <= 8192) norm_backward_kernel<T, HELD, 512, 2, 1><<<dim3(runs), 512, 0, s>>>(a, part, run);
      else if (a.features <= 16384) norm_backward_kernel<T, HELD, 1024, 2, 1><<<dim3(runs), 1024, 0, s>>>(a, part, run);
      else {
        norm_along_kernel<T, HELD><<<dim3((unsigned)a.samples), 1024, 0, s>>>(a, along);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        norm_strips_kernel<T, HELD><<<dim3((unsigned)((a.features + 2047) / 2048), runs), 256, 0, s>>>(a, along, part, run);
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (part) {
      sum_runs_kernel<<<dim3((unsigned)((a.features + 63) / 64)), 256, 0, s>>>(part, a.dgain, a.accumulate, a.features, (int)runs);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    at += kAlong;
  } while (at < all.samples);
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------
// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw 2011): each round multiplies two of the counter's words by constants, and the
// products' upper halves meet the other two words and the key, which grows by a constant a round.
__device__ inline uint4 philox(uint4 c, uint2 key) {
#pragma unroll
  for (int k = 0; k < 10; ++k) {
    const uint64_t p = (uint64_t)c.x * 0xD2511F53u, q = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(q >> 32) ^ c.y ^ key.x, (uint32_t)q, (uint32_t)(p >> 32) ^ c.w ^ key.y, (uint32_t)p);
    key.x += 0x9E3779B9u, key.y += 0xBB67AE85u;
  }
  return c;
}

// A thread takes 8 consecutive values, whose bits are one block of the generator, a workgroup a run of 256 such pieces of the whole
// tensor.  pieces: of a row; whole groups of 32 values where a checkpoint is kept.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int64_t row_first, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  const bool there = row < a.samples;
  const int col = (int)piece * kPiece, n = there ? a.features - col : 0;
  float v[kPiece], r[kPiece] = {};
  load_values(v, static_cast<const T*>(a.x) + row * a.ldx + col, n);
  if (a.residual) load_values(r, static_cast<const T*>(a.residual) + row * a.ldr + col, n);
  const uint64_t offset = a.offset + (a.more_offset ? *a.more_offset : 0);
  const uint4 bits = philox(make_uint4(piece, (uint32_t)(row_first + row), (uint32_t)offset, (uint32_t)(offset >> 32)),
                            make_uint2((uint32_t)a.seed, (uint32_t)(a.seed >> 32)));
  const uint32_t words[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int k = 0; k < kPiece; ++k) {
    const uint32_t b = k & 1 ? words[k >> 1] >> 16 : words[k >> 1] & 0xffffu;
    v[k] = (b >= a.least ? v[k] * a.factor : 0.f) + r[k];
  }
  store_values(static_cast<T*>(a.y) + row * a.ldy + col, v, n);
  if (!a.kept.codes) return;
#pragma unroll
  for (int k = 0; k < kPiece; ++k) v[k] = k < n ? widen(narrow<T>(v[k])) : 0.f;
  uint32_t w[2], byte;
  pack_codes<T>(w, v, group_largest<kPiece>(largest(v)), &byte);
  if (!there) return;
  *reinterpret_cast<uint2*>(a.kept.codes + row * ((int64_t)pieces * kPiece) + col) = make_uint2(w[0], w[1]);
  if ((piece & 3u) == 0) a.kept.exponents[row * (pieces >> 2) + (piece >> 2)] = (uint8_t)byte;
}

}  // namespace

hipError_t launch_rows_save(int type, int64_t samples, int32_t features, const void* x, int64_t ldx, Rows rows, hipStream_t s) {
  NormArgs a{};
  a.samples = samples; a.features = features; a.x = x; a.ldx = ldx; a.rows = rows;
  return by_type(type, [&](auto zero) { return run_rows<decltype(zero), false>(a, s); });
}

hipError_t launch_rows_load(int type, int64_t samples, int32_t features, Rows rows, void* x, int64_t ldx, hipStream_t s) {
  const uint32_t pieces = (uint32_t)((features + kGroup - 1) / kGroup * (kGroup / kPiece));
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    return by_slabs(samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      const Rows part{rows.codes + at * pieces * kPiece, rows.scales + at};
      rows_load_kernel<T><<<dim3(blocks), 256, 0, s>>>(static_cast<T*>(x) + at * ldx, ldx, part, n, features, pieces);
      return hipGetLastError();
    });
  });
}

hipError_t launch_rms_norm(int type, const NormArgs& a, hipStream_t s) {
  return by_type(type, [&](auto zero) { return run_rows<decltype(zero), true>(a, s); });
}

hipError_t launch_rms_norm_backward(int type, const NormBackwardArgs& a, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    return a.held.codes ? run_norm_backward<T, true>(a, s) : run_norm_backward<T, false>(a, s);
  });
}

hipError_t launch_dropout(int type, const DropoutArgs& all, hipStream_t s) {
  const uint32_t pieces = (uint32_t)(all.kept.codes ? (all.features + kGroup - 1) / kGroup * (kGroup / kPiece) : (all.features + kPiece - 1) / kPiece);
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    return by_slabs(all.samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      DropoutArgs a = all;
      a.samples = n;
      a.x = static_cast<const T*>(all.x) + at * all.ldx;
      if (a.residual) a.residual = static_cast<const T*>(all.residual) + at * all.ldr;
      a.y = static_cast<T*>(all.y) + at * all.ldy;
      if (a.kept.codes) a.kept = Codes{all.kept.codes + at * pieces * kPiece, all.kept.exponents + at * (pieces >> 2)};
      dropout_kernel<T><<<dim3(blocks), 256, 0, s>>>(a, at, pieces);
      return hipGetLastError();
    });
  });
}

}  // namespace linear
}  // namespace lqsgd
