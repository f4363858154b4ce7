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
  return absmax < __builtin_inff() ? fmaxf(absmax * (1.f / 127.f), 0x1p-126f) : __builtin_nanf("");
}
// Codes of N values, four to a word, `inverse` = 1 / step; 0 where that is NaN.  |v| inverse is 127 (1 + 2^-22) at most, which rounds to 127; the
// product is rounded before the sum that rounds it to an integer, as the definition has it.
template <int N>
__device__ inline void row_codes(uint32_t (&w)[N / 4], const float (&v)[N], float inverse) {
#pragma clang fp contract(off)
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    uint32_t q[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) q[c] = __builtin_bit_cast(uint32_t, v[4 * k + c] * inverse + 12582912.f);
    const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
    w[k] = inverse == inverse ? low | high : 0u;
  }
}

// 16 bytes of values: neighbouring threads load and store whole lines (fp32 by 32 bytes a thread stores half a line at a time, past the caches: 8192 x
// 4096 with 8-bit rows read back 45 us, not 24.6, norm with residual and checkpoint 111, not 94, backward 105, not 95).
template <typename T> constexpr int kWide = 16 / (int)sizeof(T);

// ---------------------------------------------------------------------------
// norm and 8-bit rows
// ---------------------------------------------------------------------------
// N values of a row of n from `col` on, as they lie in memory, on their way: whole words, so that 16-bit values share registers.
// ENDS (16-bit rows of N values or more): a piece that the row's end cuts, or that lies behind it, is read as the row's last N values, which get()
// moves to their places, zeros behind them.  Read value by value they are waited for one by one, and the row for them (bfloat16 4096 x 11008
// norm 42 -> 35 us, backward 90 -> 76; of 4096 x 5000 78 -> 62); fp32 values wait for nothing and have no registers for this.
template <typename T, int N, bool ENDS>
struct Raw {
  uint32_t w[N * sizeof(T) / 4];
  // PAST: past the caches.
  template <bool PAST = false>
  __device__ inline void load(const T* row, int col, int n) {
    const T* const p = row + (ENDS ? min(col, n - N) : col);
    if (ENDS || n - col >= N) {
      if constexpr (PAST) {
        typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(1)));
#pragma unroll
        for (int k = 0; k < (int)(sizeof w / 16); ++k) {
          const Words v = __builtin_nontemporal_load(reinterpret_cast<const Words*>(p) + k);
          __builtin_memcpy(w + 4 * k, &v, 16);
        }
      } else {
        __builtin_memcpy(w, p, sizeof w);
      }
    } else {
      n -= col;
#pragma unroll
      for (int k = 0; k < (int)(sizeof w / 4); ++k) {
        if constexpr (sizeof(T) == 4) {
          w[k] = k < n ? __builtin_bit_cast(uint32_t, p[k]) : 0u;
        } else {
          const uint32_t low = 2 * k < n ? __builtin_bit_cast(uint16_t, p[2 * k]) : 0u, high = 2 * k + 1 < n ? __builtin_bit_cast(uint16_t, p[2 * k + 1]) : 0u;
          w[k] = low | high << 16;
        }
      }
    }
  }
  __device__ inline void get(float (&f)[N], int col, int n) const {
    constexpr int W = sizeof w / 4;
    uint32_t x[W];
    __builtin_memcpy(x, w, sizeof x);
    const int by = col - (n - N);
    if (ENDS && by > 0) {
#pragma unroll
      for (int step = W / 2; step > 0; step >>= 1) {
        const bool on = (by / 2 & step) != 0;
#pragma unroll
        for (int k = 0; k < W; ++k) x[k] = on ? (k + step < W ? x[k + step] : 0u) : x[k];
      }
#pragma unroll
      for (int k = 0; k < W; ++k) {
        x[k] = by & 1 ? x[k] >> 16 | (k + 1 < W ? x[k + 1] << 16 : 0u) : x[k];
        x[k] = by < N ? x[k] : 0u;
      }
    }
    T v[N];
    __builtin_memcpy(v, x, sizeof v);
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = widen(v[k]);
  }
};
template <typename T> constexpr bool kEnds = sizeof(T) == 2;

// 1 / sqrt(mean + eps) in fp64: the hardware's estimate and a step of Newton's on it, which leaves 2^-40.
__device__ inline double root(double v) {
  const double y = __builtin_amdgcn_rsq(v);
  return v > 0.0 && v < __builtin_inf() ? y + 0.5 * y * (1.0 - v * y * y) : y;
}
__device__ inline double power_of_two_64(int e) { return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52); }
// Its exponent, held to what powers of two fp32 has beside their inverses.
__device__ inline int exponent_of(double v) { return min(max((int)(__builtin_bit_cast(uint64_t, v) >> 52 & 2047) - 1023, -126), 126); }

// A row to a workgroup, PIECES of 16 bytes a thread in registers, or, ROWS > 1, to each of its wavefronts; WIDE: a row of any length,
// read again for its outputs.  NORM: the norm, with what is wanted of it; otherwise 8-bit rows of x alone.  PAST: inputs past the caches.
// Bound by memory: 8192 x 4096 bfloat16 norm with residual, checkpoint and h 50 us (6.0 TB/s), with 8-bit rows 40 (5.9), the norm alone 21 (6.3), rows
// alone 18 (5.6); 4096 x 11008 norm 35 (5.1).
// Tried: workgroups that stay, keep the gain and have the next row on their way (norm alone 25 -> 29 us, single rows 0.2 us more: fewer
// wavefronts fit).
template <typename T, int PIECES, int ROWS, bool NORM, bool WIDE, bool PAST, bool ENDS = kEnds<T>>
__global__ __launch_bounds__(ROWS > 1 ? 64 * ROWS : 1024) void row_kernel(NormArgs a) {
  constexpr int N = kWide<T>;
  using R = Raw<T, N, ENDS>;
  const int threads = ROWS > 1 ? 64 : (int)blockDim.x, t = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  if (ROWS > 1 && row >= a.samples) return;
  const int n = a.features, stride = (n + kGroup - 1) / kGroup * kGroup;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const r = NORM && a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  const T* const gain = NORM ? static_cast<const T*>(a.gain) : nullptr;
  T* const h = NORM && a.h ? static_cast<T*>(a.h) + row * a.ldh : nullptr;

  // values of the row from `col` on, as the norm sees them; zeros behind its end
  auto joined = [&](float (&v)[N], const R& from, const R& more, int col) {
    from.get(v, col, n);
    if (r) {
      float m[N];
      more.get(m, col, n);
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = widen(narrow<T>(v[k] + m[k]));
    }
  };
  auto gains = [&](float (&g)[N], const R& from, int col) {
    if (gain) {
      from.get(g, col, n);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) g[k] = 1.f;
    }
  };
  double sum = 0.0;
  float most = 0.f;
  auto count_rows = [&](const float (&v)[N], const R& rg, int col) {
    if (!NORM) {
      most = __builtin_elementwise_maximum(most, largest(v));
    } else if (a.rows.codes) {
      float g[N];
      gains(g, rg, col);
#pragma unroll
      for (int k = 0; k < N; ++k) g[k] *= v[k];
      most = __builtin_elementwise_maximum(most, largest(g));
    }
  };
  auto count = [&](const float (&v)[N], const R& rg, int col) {
    if (NORM) {
#pragma unroll
      for (int k = 0; k < N; ++k) sum = __builtin_fma((double)v[k], (double)v[k], sum);
    }
    count_rows(v, rg, col);
  };

  float v[PIECES][N];
  R rx[PIECES], rr[PIECES], rg[PIECES];
  const int pieces = (n + N - 1) / N;
  // what this thread has read before
  auto again = [&](float (&v)[N], int col) {
    if (h) {
      load_values(v, h + col, n - col);           // its own; x or the residual may be gone
    } else {
      rx[0].load(x, col, n);
      if (r) rr[0].load(r, col, n);
      joined(v, rx[0], rr[0], col);
    }
  };
  if constexpr (WIDE) {
    for (int p = t; p < pieces; p += threads) {
      const int col = p * N;
      rx[0].load(x, col, n);
      if (r) rr[0].load(r, col, n);
      if (gain && a.rows.codes) rg[0].load(gain, col, n);
      joined(v[0], rx[0], rr[0], col);
      if (h) store_values(h + col, v[0], n - col);
      count(v[0], rg[0], col);
    }
  } else {
    // all of it on its way at once
#pragma unroll
    for (int p = 0; p < PIECES; ++p) rx[p].template load<PAST>(x, (t + p * threads) * N, n);
    if (r) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) rr[p].template load<PAST>(r, (t + p * threads) * N, n);
    }
    if (gain) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) rg[p].load(gain, (t + p * threads) * N, n);
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * threads) * N;
      joined(v[p], rx[p], rr[p], col);
      if (h) store_values(h + col, v[p], n - col);
      count(v[p], rg[p], col);
    }
  }
  __shared__ double sums[ROWS == 1 ? 16 : 1];
  __shared__ float mosts[ROWS == 1 ? 16 : 1];
  if (NORM) sum = over_wave(sum, Plus{});
  if (!NORM || a.rows.codes) most = over_wave(most, Larger{});
  if (ROWS == 1 && threads > 64) {
    if ((t & 63) == 0) sums[t >> 6] = sum, mosts[t >> 6] = most;
    __syncthreads();
    sum = 0.0, most = 0.f;
    for (int k = 0; k < threads >> 6; ++k) sum += sums[k], most = __builtin_elementwise_maximum(most, mosts[k]);
  }
  // Rows (all of a row's threads find the same) whose root is no normal fp32 number, or whose h gain the least step would leave without digits
  // or fp32 without a value: h is multiplied by `up`, the power of two below the root, and the rest of the root, 1 to 2, takes its place;
  // more than that, held to the largest number, only where h is 0 and eps next to nothing.
  float rstd = 1.f, up = 1.f;
  auto scaled = [&](float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] *= up;
  };
  if constexpr (NORM) {
    const double mean = sum * a.inverse + a.eps, exact = root(mean);
    rstd = (float)exact;
    if (t == 0 && a.rstd) a.rstd[row] = rstd;
    bool far = !(rstd > 0x1p-126f && rstd < 0x1p126f);
    if (a.rows.codes) far |= rstd > 1.f ? most > 0.f && most < 0x1p-119f : !(most < __builtin_inff());
    if (__builtin_expect(far && mean > 0.0 && mean < __builtin_inf(), 0)) {
      const int e = exponent_of(exact);
      rstd = fminf((float)(exact * power_of_two_64(-e)), 0x1.fffffep127f);
      up = power_of_two(e);
      if constexpr (!WIDE) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) scaled(v[p]);
      }
      if (a.rows.codes) {
        most = 0.f;
        if constexpr (WIDE) {
          for (int p = t; p < pieces; p += threads) {
            again(v[0], p * N);
            if (gain) rg[0].load(gain, p * N, n);
            scaled(v[0]);
            count_rows(v[0], rg[0], p * N);
          }
        } else {
#pragma unroll
          for (int p = 0; p < PIECES; ++p) count_rows(v[p], rg[p], (t + p * threads) * N);
        }
        most = over_wave(most, Larger{});
        if (ROWS == 1 && threads > 64) {
          __syncthreads();                        // all have read the first ones
          if ((t & 63) == 0) mosts[t >> 6] = most;
          __syncthreads();
          most = 0.f;
          for (int k = 0; k < threads >> 6; ++k) most = __builtin_elementwise_maximum(most, mosts[k]);
        }
      }
    }
  }
  const float step = row_step(most), inverse = 1.f / step;
  if (t == 0 && a.rows.codes) a.rows.scales[row] = NORM ? step * rstd : step;
  auto write = [&](const float (&v)[N], const R& rg, int col) {
    float g[N];
    gains(g, rg, col);
    if (a.rows.codes) {
      float q[N];
#pragma unroll
      for (int k = 0; k < N; ++k) q[k] = NORM ? v[k] * g[k] : v[k];
      uint32_t w[N / 4];
      row_codes<N>(w, q, inverse);
      if (col < stride) __builtin_memcpy(__builtin_assume_aligned(a.rows.codes + row * stride + col, N), w, N);
    }
    if (!NORM || (!a.y && !a.kept.codes)) return;
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] *= v[k] * rstd;
    if (a.y) store_values(static_cast<T*>(a.y) + row * a.ldy + col, g, n - col);
    if (!a.kept.codes) return;
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] = widen(narrow<T>(g[k]));
    uint32_t w[N / 4], byte;
    pack_codes<T>(w, g, group_largest<N>(largest(g)), &byte);
    if (col >= stride) return;
    __builtin_memcpy(__builtin_assume_aligned(a.kept.codes + row * stride + col, N), w, N);
    if (col % kGroup == 0) a.kept.exponents[row * (stride / kGroup) + col / kGroup] = (uint8_t)byte;
  };
  if constexpr (WIDE) {
    // whole wavefronts go round together: lanes exchange what a group's largest value is
    for (int p = t; p < (pieces + 63) / 64 * 64; p += threads) {
      const int col = p * N;
      if (gain) rg[0].load(gain, col, n);
      again(v[0], col);
      scaled(v[0]);
      write(v[0], rg[0], col);
    }
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) write(v[p], rg[p], (t + p * threads) * N);
  }
}

// Inputs of this size and more are read past the caches (bfloat16 8192 x 4096: norm with residual and checkpoint 58.8 -> 53.3 us, rows
// 19.7 -> 18.1, dropout with residual 38.4 -> 33.9; of half the size the norm 25.4 -> 30.2), but not by the norm and dropout of a single input
// (25.6 -> 29.5, 24.3 -> 25.7).
constexpr int64_t kPastBytes = int64_t(1) << 26;

template <typename T, bool NORM, bool PAST>
hipError_t run_rows(const NormArgs& all, hipStream_t s) {
  // a launch has fewer than 2^32 threads
  constexpr int64_t kSlab = int64_t(1) << 21;
  const int64_t stride = (all.features + kGroup - 1) / kGroup * kGroup;
  const int pieces = (all.features + kPiece - 1) / kPiece;
  for (int64_t at = 0; at < all.samples; at += kSlab) {
    NormArgs a = all;
    a.samples = std::min(kSlab, all.samples - at);
    a.inverse = 1.0 / a.features;
    a.x = static_cast<const T*>(all.x) + at * all.ldx;
    if (a.residual) a.residual = static_cast<const T*>(all.residual) + at * all.ldr;
    if (a.h) a.h = static_cast<T*>(all.h) + at * all.ldh;
    if (a.y) a.y = static_cast<T*>(all.y) + at * all.ldy;
    if (a.rstd) a.rstd += at;
    if (a.kept.codes) a.kept = Codes{all.kept.codes + at * stride, all.kept.exponents + at * (stride / kGroup)};
    if (a.rows.codes) a.rows = Rows{all.rows.codes + at * stride, all.rows.scales + at};
    const unsigned n = (unsigned)a.samples;
    constexpr int Q = kPiece / kWide<T>;
    auto threads = [&](int each) { return dim3((unsigned)((pieces + 64 * each - 1) / (64 * each)) * 64); };
    // Threads take 1, 2 or 4 times 8 values.  The norm by 8 where that goes: the more wavefronts, the sooner a row is there (1 x 4096 by 16 3.3 us,
    // by 8 3.0; fp32 4096 x 5000 30.8 and 28.2).  Many rows by 16, which leaves more of them on a CU (8192 x 4096 21.1 us, by 8
    // 25.1; 4096 x 7000 20.5 and 30.4; but with a checkpoint, 8192 x 4096 50.8 and 49.5; fp32 4096 x 7000 43.5 and 50.4, with a checkpoint 92.9
    // and 90.4), and from 12 wavefronts on by 32 (4096 x 13500 45.6 us, by 16 53.8; 4096 x 12000 41.4 and 38.8; fp32 4096 x 13500 89 and 104).  All others of more than 14 wavefronts by 32, so that two fit a CU (2000 x 16384 28.8
    // us, not 32.9).
    const bool many = NORM && a.samples > 512, kept = a.kept.codes != nullptr;
    const bool two = many && (Q == 2 ? pieces > 768 && !kept : pieces > (kept ? 512 : 256));
    // few short fp32 rows by 4 (300 x 513 with a checkpoint 4.0 us, by 8 4.6; 1 x 4096 3.8 and 3.7)
    if (Q == 2 && NORM && a.samples <= 512 && pieces <= 256) row_kernel<T, 1, 1, NORM, false, PAST><<<dim3(n), dim3((unsigned)(2 * pieces + 63) / 64 * 64), 0, s>>>(a);
    else if (pieces == 1) row_kernel<T, Q, 4, NORM, false, PAST, false><<<dim3((n + 3) / 4), 256, 0, s>>>(a);
    else if (pieces <= 64) row_kernel<T, Q, 4, NORM, false, PAST><<<dim3((n + 3) / 4), 256, 0, s>>>(a);
    else if (NORM && pieces <= 1024 && !two) row_kernel<T, Q, 1, NORM, false, PAST><<<dim3(n), threads(1), 0, s>>>(a);
    else if (pieces <= 2 * 64 * (many ? 12 : 14)) row_kernel<T, 2 * Q, 1, NORM, false, PAST><<<dim3(n), threads(2), 0, s>>>(a);
    else if (pieces <= 4096) row_kernel<T, 4 * Q, 1, NORM, false, PAST><<<dim3(n), threads(4), 0, s>>>(a);
    else row_kernel<T, 1, 1, NORM, true, false><<<dim3(n), 1024, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T, bool NORM>
hipError_t run_rows(const NormArgs& a, hipStream_t s) {
  const bool past = (!NORM || a.residual) && a.samples * a.features * (int64_t)sizeof(T) >= kPastBytes;
  return past ? run_rows<T, NORM, true>(a, s) : run_rows<T, NORM, false>(a, s);
}

// 8192 x 4096 bfloat16 16.6 us, 6.1 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void rows_load_kernel(T* x, int64_t ldx, Rows rows, int64_t samples, int features, uint32_t pieces) {
  constexpr int N = kWide<T>;
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  if (row >= samples) return;
  int8_t q[N];
  __builtin_memcpy(q, __builtin_assume_aligned(rows.codes + row * ((int64_t)pieces * N) + piece * N, N), N);
  const float scale = rows.scales[row];
  float v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = (float)q[k] * scale;
  store_values(x + row * ldx + piece * N, v, features - (int)(piece * N));
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

// A workgroup takes a row or, ROWS > 1, one to each of its wavefronts at a time, those that run together neighbouring ones; a thread keeps its
// columns' gain and sums, and, but for the widest rows, has the next row's values on their way.  dgain: `part`, runs x `stride`, where it is
// wanted.  dot and sums are fp32: what is added up has been rounded to fp32 once and is of the output's size.
// Bound by memory: 8192 x 4096 bfloat16 with dh 44 us (6.1 TB/s) without dgain; the runs' sums, 8 MiB, and norm_gain_kernel take 8 more.  Rows of
// 8193 to 12288 features 69 us (4096 x 11008, 5.2 TB/s; without the next row on its way 76), up to 16384 4.5 TB/s, of 4097 to 6144, whose workgroups
// are two a CU with as many runs, 3.7 to 4 (4096 x 5000 43.8 us, 35.3 without dgain).  From a checkpoint 3.5 to 4.8 (50.5 us, 4096 x 7000 57.4, 47.2 from the
// tensor): codes by 8 bytes and exponents by one a lane, through the caches.  Tried: two rows on their way (no gain).
template <typename T, bool HELD, int PIECES, int ROWS, int MOST, bool PAST, bool ENDS = kEnds<T>>
__global__ __launch_bounds__(MOST, MOST == 768 && PIECES == 1 ? 6 : 1) void norm_backward_kernel(NormBackwardArgs a, float* part, int stride) {
  const int threads = ROWS > 1 ? 64 : (int)blockDim.x, t = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x, n = a.features;
  const int slot = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const int64_t step = (int64_t)gridDim.x * ROWS, last = a.samples;
  // (rows of a wavefront each are as fast by 32 bytes, and the sooner there where they are few: 64 x 1024 fp32 7.0 us, by 16 7.3)
  constexpr int N = ROWS > 1 ? kPiece : kWide<T>;
  using R = Raw<T, N, ENDS>;
  struct Held { uint32_t w[N / 4]; };
  struct Row {
    R dy[PIECES], dh[PIECES];
    std::conditional_t<HELD, Held, R> h[PIECES];
    uint32_t exps[HELD ? PIECES : 1];
    float rstd;
  };
  const int groups = (n + kGroup - 1) / kGroup;
  auto ask = [&](Row& q, int64_t row) {
    q.rstd = a.rstd[row];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * threads) * N;
      q.dy[p].template load<PAST>(static_cast<const T*>(a.dy) + row * a.lddy, col, n);
      if constexpr (HELD) {
        const int in = min(col, groups * kGroup - N);                  // codes go on to the end of their group
        __builtin_memcpy(&q.h[p], __builtin_assume_aligned(a.held.codes + row * ((int64_t)groups * kGroup) + in, N), N);
        q.exps[p] = a.held.exponents[row * groups + in / kGroup];
      } else {
        q.h[p].template load<PAST>(static_cast<const T*>(a.h) + row * a.ldh, col, n);
      }
      if (a.dh) q.dh[p].template load<PAST>(static_cast<const T*>(a.dh) + row * a.lddh, col, n);
    }
  };
  constexpr bool kNext = MOST <= 768;              // 1024 threads have no registers for it (2048 x 14000 60 -> 78 us)
  R gain[PIECES];
  float sums[PIECES][N] = {};
  Row now, next;
  int64_t row = (int64_t)blockIdx.x * ROWS + slot;
  if (kNext && row < last) ask(now, row);
  if (a.gain) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) gain[p].load(static_cast<const T*>(a.gain), (t + p * threads) * N, n);
  }
  __shared__ float dots[2][16];
  for (int turn = 0; row < last; row += step, turn ^= 1) {
    if (!kNext) ask(now, row);
    else if (row + step < last) ask(next, row + step);
    float dy[PIECES][N], h[PIECES][N], dot = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = (t + p * threads) * N;
      now.dy[p].get(dy[p], col, n);
      if constexpr (HELD) {
        const float f = factor_of(now.exps[p]);
        const int left = n - col;                                          // behind the row's end dy is 0, and so is what is made of h
#pragma unroll
        for (int k = 0; k < N; ++k) h[p][k] = k < left ? (float)(int8_t)(now.h[p].w[k / 4] >> (8 * (k % 4))) * f : 0.f;
      } else {
        now.h[p].get(h[p], col, n);
      }
      float g[N];
      if (a.gain) {
        gain[p].get(g, col, n);
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) g[k] = 1.f;
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        h[p][k] *= now.rstd;
        sums[p][k] = fmaf(dy[p][k], h[p][k], sums[p][k]);
        dy[p][k] *= g[k];
        dot = fmaf(dy[p][k], h[p][k], dot);
      }
    }
    if (a.dx) {
      dot = over_wave(dot, Plus{});
      if (ROWS == 1 && threads > 64) {
        if ((t & 63) == 0) dots[turn][t >> 6] = dot;
        __syncthreads();
        dot = 0.f;
        for (int k = 0; k < threads >> 6; ++k) dot += dots[turn][k];
      }
      const float along = dot / (float)n;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int col = (t + p * threads) * N;
        float d[N] = {};
        if (a.dh) now.dh[p].get(d, col, n);
#pragma unroll
        for (int k = 0; k < N; ++k) d[k] = fmaf(now.rstd, fmaf(-h[p][k], along, dy[p][k]), d[k]);
        store_values(static_cast<T*>(a.dx) + row * a.lddx + col, d, n - col);
      }
    }
    if (kNext) now = next;
  }
  if (!part) return;
  float* const out = part + (int64_t)blockIdx.x * stride;
  const bool whole = a.arrived != nullptr && gridDim.x == 1, joins = ROWS > 1 && a.arrived != nullptr;
  auto put = [&](int f, float v) {
    if (f >= n) return;
    if (whole) a.dgain[f] = a.accumulate ? a.dgain[f] + v : v;
    else if (joins) __hip_atomic_store(out + f, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else out[f] = v;
  };
  if constexpr (ROWS > 1) {
    __shared__ float all[ROWS][PIECES * 64 * N];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int k = 0; k < N; ++k) all[slot][(t + p * threads) * N + k] = sums[p][k];
    __syncthreads();
    for (int f = threadIdx.x; f < n; f += 64 * ROWS) {
      float total = 0.f;
#pragma unroll
      for (int k = 0; k < ROWS; ++k) total += all[k][f];
      put(f, total);
    }
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      int f = (t + p * threads) * N;
      asm volatile("" : "+v"(f));                                          // found anew: what would be kept of it through the loop goes to scratch in its stead
      if (f >= n) continue;                                                // `stride` has room for whole pieces
      if (whole) {
#pragma unroll
        for (int k = 0; k < N; ++k) put(f + k, sums[p][k]);
      } else {
        __builtin_memcpy(__builtin_assume_aligned(out + f, 16), sums[p], sizeof sums[p]);
      }
    }
  }
  if constexpr (ROWS > 1) {
    if (!joins || whole) return;
    // The workgroup that comes last joins the runs' sums, in the runs' order, whichever it is.  They are stored and read with agent-scope
    // atomics, which go past the caches that the XCDs do not share: every store has arrived when vmcnt says so, and the barrier puts all of the
    // workgroup's before its count.
    __shared__ int last_one;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      last_one = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
      if (last_one) __hip_atomic_store(a.arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);        // for the next launch
    }
    __syncthreads();
    if (!last_one) return;
    // two columns and 16 runs at a time
    for (int f = 2 * (int)threadIdx.x; f < n; f += 2 * (int)blockDim.x) {
      float total[2] = {};
      for (int k = 0; k < (int)gridDim.x; k += 16) {
        uint64_t x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u)
          x[u] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(part + (int64_t)min(k + u, (int)gridDim.x - 1) * stride + f), __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          float v[2];
          __builtin_memcpy(v, &x[u], sizeof v);
#pragma unroll
          for (int c = 0; c < 2; ++c) total[c] += k + u < (int)gridDim.x ? v[c] : 0.f;
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (f + c < n) a.dgain[f + c] = a.accumulate ? a.dgain[f + c] + total[c] : total[c];
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
__global__ __launch_bounds__(256) void norm_strips_kernel(NormBackwardArgs a, const float* along, float* part, int stride, int64_t run) {
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
    if (col + k < n) part[(int64_t)blockIdx.y * stride + col + k] = sums[k];
}

// dgain from the runs' sums: a workgroup adds up 16 columns, 64 runs at a time, in an order of its own that is always the same.  512 runs x 4096
// features 4.6 us, most of it the launch and a round trip to memory.
__global__ __launch_bounds__(256) void norm_gain_kernel(const float* part, float* dgain, int accumulate, int n, int stride, int runs) {
  __shared__ float sums[64][17];
  const int col = (int)blockIdx.x * 16 + (threadIdx.x & 3) * 4, slot = threadIdx.x >> 2;
  float s[4] = {};
#pragma unroll 8
  for (int k = slot; k < runs; k += 64) {
    const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)k * stride + col);
    s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) sums[slot][(threadIdx.x & 3) * 4 + k] = s[k];
  __syncthreads();
  // 16 threads a column, four runs' sums each
  const int f = threadIdx.x >> 4, part4 = threadIdx.x & 15;
  float total = (sums[part4][f] + sums[part4 + 16][f]) + (sums[part4 + 32][f] + sums[part4 + 48][f]);
#pragma unroll
  for (int k = 8; k > 0; k >>= 1) total += __shfl_xor(total, k, 16);
  const int at = (int)blockIdx.x * 16 + f;
  if (part4 == 0 && at < n) dgain[at] = accumulate ? dgain[at] + total : total;
}

constexpr int64_t kAlong = int64_t(1) << 21;              // rows at a time; wide ones' means lie in front of the parts in the workspace
constexpr int64_t kPartFloats = (int64_t)(kWorkspaceBytes / 4) - kAlong;

template <typename T, bool HELD, bool PAST>
hipError_t run_norm_backward(const NormBackwardArgs& all, hipStream_t s) {
  float* const along = static_cast<float*>(all.workspace);
  float* const parts = along + kAlong;
  constexpr int Q = kPiece / kWide<T>;
  const int64_t groups = (all.features + kGroup - 1) / kGroup;
  const int pieces = (all.features + kPiece - 1) / kPiece, stride = (all.features + 15) / 16 * 16;
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
    // A row takes a workgroup about 1.25 us, and a run's sums their time to be written, read and joined: the rows of a run grow with the
    // root of their number (bfloat16, us: 512 x 4096 by 1, 2, 4, 8 rows 16.7, 13.3, 13.4, 17.9; 8192 x 4096 by 4, 8, 16, 32 69.8, 65.9, 56.6, 63.9;
    // 8192 x 512, four wavefronts a row each, by 4, 8, 16, 32 17.4, 12.8, 11.9, 12.3).
    const int waves = pieces <= 128 ? 4 : std::min(16, (pieces + 127) / 128), rows = pieces <= 128 ? 4 : 1;
    const bool wide = pieces > 2 * 1024;
    int64_t run = wide ? std::max<int64_t>(1, a.samples * a.features / (1024 * 2048)) : rows;
    while (!wide && (run / rows + 1) * (run / rows + 1) * (rows > 1 ? 512 : 32) <= a.samples) run += rows;
    // one piece a thread where two such workgroups of up to 12 wavefronts fit a CU, which fp32 has no registers for (by two pieces and
    // one workgroup: bfloat16 4096 x 4608 46 us, not 40, 4096 x 6000 55, not 49; fp32 by one piece 81, by two 62)
    const bool single = kEnds<T> && pieces > 512 && pieces <= 768;
    // no more runs than workgroups run together: 12 wavefronts a CU, but a workgroup of five or more has it alone (its wavefronts lie on the four
    // SIMDs unevenly)
    const int64_t together = 256 * (waves <= 4 ? 12 / waves : single ? 2 : 1);
    if (!wide && run * together < a.samples) run = (a.samples + together * rows - 1) / (together * rows) * rows;
    const int64_t least = (a.samples + kPartFloats / stride - 1) / (kPartFloats / stride);
    if (run < least) run = (least + rows - 1) / rows * rows;
    // as many runs for each CU (fp32 4096 x 5000 85 -> 75 us)
    if (!wide && a.samples > 256 * run) {
      const int64_t even = ((a.samples + run - 1) / run + 255) / 256 * 256;
      run = ((a.samples + even - 1) / even + rows - 1) / rows * rows;
      if (run < least) run = (least + rows - 1) / rows * rows;
    }
    const unsigned runs = (unsigned)((a.samples + run - 1) / run);
    float* const part = a.dgain ? parts : nullptr;
    // One run's sums, and few that wavefronts with a row each have made, are joined in the kernel itself: no second launch, 3 us less on the host.
    // The last workgroup does that by itself, 16 runs at a time (us, itself / second launch, bfloat16: 64 x 256 4.8 / 5.4, 64 x 1024 6.5 / 6.0,
    // 256 x 64 6.8 / 5.4; not so 512 x 32 9.5 / 5.4, 8192 x 16 28.4 / 8.3, 300 x 513 11.1 / 6.8, nor runs of a row to a workgroup, 2 x 2048 10.1 / 5.5).
    const bool joins = part && !wide && a.samples > 0 && (runs == 1 || (rows > 1 && runs <= 64)) && (int64_t)runs * stride <= int64_t(1) << 14;
    if (!joins) a.arrived = nullptr;
    if (a.samples > 0) {
      // 8 features or fewer: there may be no whole piece to read
      if (pieces == 1) norm_backward_kernel<T, HELD, 1, 4, 256, PAST, false><<<dim3(runs), 256, 0, s>>>(a, part, stride);
      else if (pieces <= 64) norm_backward_kernel<T, HELD, 1, 4, 256, PAST><<<dim3(runs), 256, 0, s>>>(a, part, stride);
      else if (pieces <= 128) norm_backward_kernel<T, HELD, 2, 4, 256, PAST><<<dim3(runs), 256, 0, s>>>(a, part, stride);
      else if (waves <= 4) norm_backward_kernel<T, HELD, 2 * Q, 1, 256, PAST><<<dim3(runs), dim3((unsigned)waves * 64), 0, s>>>(a, part, stride);
      else if (single) {
        if constexpr (kEnds<T>) norm_backward_kernel<T, HELD, 1, 1, 768, PAST><<<dim3(runs), dim3((unsigned)(pieces + 63) / 64 * 64), 0, s>>>(a, part, stride);
      } else if (waves <= 8) norm_backward_kernel<T, HELD, 2 * Q, 1, 512, PAST><<<dim3(runs), dim3((unsigned)waves * 64), 0, s>>>(a, part, stride);
      else if (waves <= 12) norm_backward_kernel<T, HELD, 2 * Q, 1, 768, PAST><<<dim3(runs), dim3((unsigned)waves * 64), 0, s>>>(a, part, stride);
      else if (!wide) norm_backward_kernel<T, HELD, 2 * Q, 1, 1024, PAST><<<dim3(runs), dim3((unsigned)waves * 64), 0, s>>>(a, part, stride);
      else {
        norm_along_kernel<T, HELD><<<dim3((unsigned)a.samples), 1024, 0, s>>>(a, along);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        norm_strips_kernel<T, HELD><<<dim3((unsigned)((a.features + 2047) / 2048), runs), 256, 0, s>>>(a, along, part, stride, run);
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (part && !joins) {
      norm_gain_kernel<<<dim3((unsigned)((a.features + 15) / 16)), 256, 0, s>>>(part, a.dgain, a.accumulate, a.features, stride, (int)runs);
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

// A thread takes 16 bytes: 8 values, whose bits are one block of the generator, or in fp32 half of them (two threads make the block: a
// thread that takes all 8 stores half lines).  Bound by memory: 8192 x 4096 bfloat16 with residual 33.9 us (5.9 TB/s), with a checkpoint too 40.4 (5.8).
// A workgroup has a run of 256 such pieces of the whole tensor.  pieces: of a row; whole groups of 32 values where a checkpoint is kept.
template <typename T, bool PAST, bool ENDS>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int64_t row_first, uint32_t pieces) {
  constexpr int N = kWide<T>, kParts = 8 / N, kGroupPieces = kGroup / N;
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  const bool there = row < a.samples;
  const int col = (int)piece * N;
  float v[N], r[N] = {};
  Raw<T, N, ENDS> rx, rr;
  // threads behind the last row read that one's
  const int64_t from = there ? row : a.samples - 1;
  rx.template load<PAST>(static_cast<const T*>(a.x) + from * a.ldx, col, a.features);
  if (a.residual) rr.template load<PAST>(static_cast<const T*>(a.residual) + from * a.ldr, col, a.features);
  const uint64_t offset = a.offset + (a.more_offset ? *a.more_offset : 0);
  const uint4 bits = philox(make_uint4(piece / kParts, (uint32_t)(row_first + row), (uint32_t)offset, (uint32_t)(offset >> 32)),
                            make_uint2((uint32_t)a.seed, (uint32_t)(a.seed >> 32)));
  const bool high = kParts > 1 && piece % kParts;
  const uint32_t words[4] = {high ? bits.z : bits.x, high ? bits.w : bits.y, bits.z, bits.w};
  rx.get(v, col, a.features);
  if (a.residual) rr.get(r, col, a.features);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t b = k & 1 ? words[k >> 1] >> 16 : words[k >> 1] & 0xffffu;
    v[k] = (b >= a.least ? v[k] * a.factor : 0.f) + r[k];
  }
  const int n = there ? a.features - col : 0;
  store_values(static_cast<T*>(a.y) + row * a.ldy + col, v, n);
  if (!a.kept.codes) return;
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = k < n ? widen(narrow<T>(v[k])) : 0.f;
  uint32_t w[N / 4], byte;
  pack_codes<T>(w, v, group_largest<N>(largest(v)), &byte);
  if (!there) return;
  __builtin_memcpy(__builtin_assume_aligned(a.kept.codes + row * ((int64_t)pieces * N) + col, N), w, N);
  if (piece % kGroupPieces == 0) a.kept.exponents[row * (pieces / kGroupPieces) + piece / kGroupPieces] = (uint8_t)byte;
}

}  // namespace

hipError_t launch_rows_save(int type, int64_t samples, int32_t features, const void* x, int64_t ldx, Rows rows, hipStream_t s) {
  NormArgs a{};
  a.samples = samples; a.features = features; a.x = x; a.ldx = ldx; a.rows = rows;
  return by_type(type, [&](auto zero) { return run_rows<decltype(zero), false>(a, s); });
}

hipError_t launch_rows_load(int type, int64_t samples, int32_t features, Rows rows, void* x, int64_t ldx, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    const uint32_t pieces = (uint32_t)((features + kGroup - 1) / kGroup * (kGroup / kWide<T>));
    return by_slabs(samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      const Rows part{rows.codes + at * pieces * kWide<T>, rows.scales + at};
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
    // by values: bfloat16 of 2^25 bytes 31.3 us, past the caches 32.6, of 5.6e7 59 and 47; fp32 of 4.9e7 bytes 45.5 and 48.7, of 2^26 the same
    const bool past = a.samples * a.features > int64_t(1) << 24;
    if (a.held.codes) return past ? run_norm_backward<T, true, true>(a, s) : run_norm_backward<T, true, false>(a, s);
    return past ? run_norm_backward<T, false, true>(a, s) : run_norm_backward<T, false, false>(a, s);
  });
}

hipError_t launch_dropout(int type, const DropoutArgs& all, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    constexpr int N = kWide<T>;
    const uint32_t pieces = (uint32_t)(all.kept.codes ? (all.features + kGroup - 1) / kGroup * (kGroup / N) : (all.features + N - 1) / N);
    const bool past = all.residual && all.samples * all.features * (int64_t)sizeof(T) >= kPastBytes;
    return by_slabs(all.samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      DropoutArgs a = all;
      a.samples = n;
      a.x = static_cast<const T*>(all.x) + at * all.ldx;
      if (a.residual) a.residual = static_cast<const T*>(all.residual) + at * all.ldr;
      a.y = static_cast<T*>(all.y) + at * all.ldy;
      if (a.kept.codes) a.kept = Codes{all.kept.codes + at * pieces * N, all.kept.exponents + at * (pieces / (kGroup / N))};
      if (all.features < N) dropout_kernel<T, false, false><<<dim3(blocks), 256, 0, s>>>(a, at, pieces);
      else if (past) dropout_kernel<T, true, kEnds<T>><<<dim3(blocks), 256, 0, s>>>(a, at, pieces);
      else dropout_kernel<T, false, kEnds<T>><<<dim3(blocks), 256, 0, s>>>(a, at, pieces);
      return hipGetLastError();
    });
  });
}

}  // namespace linear
}  // namespace lqsgd
