// What the gfx950 kernels of the linear layer and of its neighbours share: types, checkpoints' codes, activations, values from and to
// memory, and how a tile of sums leaves the matrix instructions' layout.
#pragma once

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

__device__ inline float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// The largest magnitude, NaN if one is (v_maximum3_f32: two values an instruction).
template <int N>
__device__ inline float largest(const float (&v)[N]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) m = __builtin_elementwise_maximum(m, fabsf(v[k]));
  return m;
}
// The largest of the 32 / N neighbouring lanes that share a group: lanes exchanged within fours and, for N = 4, within eights.
template <int N>
__device__ inline float group_largest(float m) {
  static_assert(N == 8 || N == 4);
  auto of = [](float v, auto control) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
  };
  m = __builtin_elementwise_maximum(m, of(m, std::integral_constant<int, 0xb1>{}));        // lane ^ 1
  m = __builtin_elementwise_maximum(m, of(m, std::integral_constant<int, 0x4e>{}));        // lane ^ 2
  if (N == 4) m = __builtin_elementwise_maximum(m, of(m, std::integral_constant<int, 0x141>{}));   // 7 - lane
  return m;
}
// e of a group from its largest magnitude.  absmax = m 2^E, 1 <= m < 2, takes e = E - 6, or E - 5 from 127.5 2^(E-6) on: adding 2^-7
// of the mantissa carries into the exponent there.
template <typename T>
__device__ inline int group_exponent(float absmax) {
  const int e = (int)((__builtin_bit_cast(uint32_t, absmax) + 0x10000u) >> 23) - 133;
  return min(max(e, Exponents<T>::lo), Exponents<T>::hi);
}
// What a code's factor is: 2^e, NaN for byte 255.
__device__ inline float factor_of(uint32_t byte) {
  return byte == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
}

__device__ inline void decode(float (&v)[8], uint2 w, float f) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k] = (float)(int8_t)(w.x >> (8 * k)) * f;
    v[4 + k] = (float)(int8_t)(w.y >> (8 * k)) * f;
  }
}

// Phi(-|z|) = erfc(x) / 2, x = |z| / sqrt 2.  With t = 1 / (1 + 0.45 x), erfc(x) exp(x^2) = t P(t); P of degree 9 is a fit that makes the
// largest relative error over all x >= 0 least, 3.2e-8, and the sizes of its terms add up to 1.8 times its value at most, so that the sum
// loses no digits: relative to its own size the tail is as good as exp(-z^2 / 2), for every type.  (A fit to 1.5e-7 of 1 has five terms
// less, but is 1e-4 of the tail off at z = -3 and 1e-2 at -8, and 8.5e-8 of normal fp32 values' gelu, this one 3.8e-8, as a rounded erf
// is; 4096 x 4096 -> 11008 with gelu 464 us with it, 468 with this one.)  `density`: exp(-z^2 / 2).
__device__ inline float normal_tail(float z, float* density) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.31819805f, fabsf(z), 1.f));
  const float g = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  float p = fmaf(-0.0207054847f, t, 0.0953871373f);
  p = fmaf(p, t, -0.150369752f);
  p = fmaf(p, t, 0.071277874f);
  p = fmaf(p, t, -0.0112238711f);
  p = fmaf(p, t, 0.0599907898f);
  p = fmaf(p, t, 0.0876229301f);
  p = fmaf(p, t, 0.114136158f);
  p = fmaf(p, t, 0.126941565f);
  p = fmaf(p, t, 0.126942661f);
  *density = g;
  return p * t * g;
}
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }

// act'(z) of gelu = Phi(z) + z phi(z), at -|z|, and 1 less that for z > 0.
__device__ inline float gelu_slope(float z) {
  float g;
  const float tail = normal_tail(z, &g), s = fmaf(-0.39894228040143268f * fabsf(z), g, tail);
  return z > 0.f ? 1.f - s : s;
}
// act'(z) of silu = s (1 + z (1 - s)), s = sigmoid(z), at -|z| likewise: no difference of nearly equal numbers, so that the
// slope is right relative to its size where it goes to 0 and to a few units in the last place where it goes to 1 (from s itself z (1 - s)
// is off by z units).  exp(-|z|) as the square of its root: what is left of z exp(z) where exp(z) itself is below the floats stays.
__device__ inline float silu_slope(float z) {
  const float x = fabsf(z), root = __builtin_amdgcn_exp2f(-0.72134752044448170f * x);
  const float c = __builtin_amdgcn_rcpf(fmaf(root, root, 1.f));           // 1 - s
  const float t = root * (c * fmaf(-x, c, 1.f)) * root;
  return z > 0.f ? 1.f - t : t;
}

// One branch for all values: which activation it is, is the same for the whole launch.
template <int N>
__device__ inline void activate_all(float (&v)[N], int act) {
  if (act == kRelu) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = v[k] < 0.f ? 0.f : v[k];           // keeps NaN
  } else if (act == kGelu) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float g;
      const float tail = normal_tail(v[k], &g);
      v[k] *= v[k] > 0.f ? 1.f - tail : tail;
    }
  } else if (act == kSilu) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] *= sigmoid(v[k]);
  }
}
// d *= act'(z)
template <int N>
__device__ inline void times_slope(float (&d)[N], const float (&z)[N], int act) {
  if (act == kRelu) {
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] *= z[k] > 0.f ? 1.f : z[k] == z[k] ? 0.f : z[k];
  } else if (act == kGelu) {
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] *= gelu_slope(z[k]);
  } else if (act == kSilu) {
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] *= silu_slope(z[k]);
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
// BYTES to memory of any alignment, past the caches: nothing here reads its outputs again, and what does soon after finds them no
// later (8192 x 4096 values: loading a checkpoint 20 -> 16 us, that and an addition that reads them 39.8 -> 38.0; small tensors alike).
// Not so the codes of checkpoints, which fit the memory-side cache longer (saving and loading 8192 x 4096 values 34 us, past it 40).
template <int BYTES>
__device__ inline void stream_out(void* p, const void* from) {
  constexpr int kWords = BYTES >= 16 ? 4 : BYTES / 4;
  typedef uint32_t Words __attribute__((ext_vector_type(kWords), aligned(1)));
#pragma unroll
  for (int k = 0; k < BYTES / 4 / kWords; ++k) {
    Words w;
    __builtin_memcpy(&w, static_cast<const char*>(from) + 16 * k, sizeof w);
    __builtin_nontemporal_store(w, reinterpret_cast<Words*>(p) + k);
  }
}
template <int N, typename T>
__device__ inline void store_values(T* p, const float (&v)[N], int n) {
  T t[N];
  if constexpr (sizeof t >= 4) {
    if (n >= N) {
#pragma unroll
      for (int k = 0; k < N; ++k) t[k] = narrow<T>(v[k]);
      stream_out<sizeof t>(p, t);
      return;
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < n) p[k] = narrow<T>(v[k]);
}

// N values of one group quantised and packed, four to a word; `absmax` is the whole group's.  v 2^-e + 1.5 2^23 rounds to the
// nearest integer, ties to even, and has it in its low byte; only the largest e leaves values that have to be held to 127.
template <typename T, int N>
__device__ inline void pack_codes(uint32_t (&w)[N / 4], const float (&v)[N], float absmax, uint32_t* byte) {
  const bool finite = absmax < __builtin_inff();
  const int e = group_exponent<T>(absmax);
  const float inv = power_of_two(-e), most = e == Exponents<T>::hi ? 127.f : 128.f;
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    uint32_t q[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float x = __builtin_amdgcn_fmed3f(v[4 * k + c] * inv, -most, most);
      q[c] = __builtin_bit_cast(uint32_t, x + 12582912.f);
    }
    const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
    w[k] = finite ? low | high : 0u;
  }
  *byte = finite ? (uint32_t)(e + 127) : 255u;
}

constexpr int kPiece = 8;                         // values that a thread takes at once

// ---------------------------------------------------------------------------
// a wavefront's lanes put together
// ---------------------------------------------------------------------------
// What all 64 lanes have, put together by `op` (commutative): every lane gets the same bits.  Lanes are exchanged within 4, 8 and 16,
// then rows of 16 and halves of 32 change places.
template <typename V, typename Op>
__device__ inline V over_wave(V v, Op op) {
  constexpr int kWords = sizeof(V) / 4;
  auto moved = [&](auto control) {
    uint32_t w[kWords];
    __builtin_memcpy(w, &v, sizeof v);
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = (uint32_t)__builtin_amdgcn_mov_dpp((int)w[k], decltype(control)::value, 0xf, 0xf, true);
    V o;
    __builtin_memcpy(&o, w, sizeof o);
    return o;
  };
  v = op(v, moved(std::integral_constant<int, 0xb1>{}));           // lane ^ 1
  v = op(v, moved(std::integral_constant<int, 0x4e>{}));           // lane ^ 2
  v = op(v, moved(std::integral_constant<int, 0x141>{}));          // 7 - lane, of 8
  v = op(v, moved(std::integral_constant<int, 0x140>{}));          // 15 - lane, of 16
  auto halves = [&](auto swap) {
    uint32_t w[kWords], a[kWords], b[kWords];
    __builtin_memcpy(w, &v, sizeof v);
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const auto r = swap(w[k]);
      a[k] = r[0], b[k] = r[1];
    }
    V x, y;
    __builtin_memcpy(&x, a, sizeof x);
    __builtin_memcpy(&y, b, sizeof y);
    return op(x, y);
  };
  v = halves([](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
  return halves([](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
}
struct Plus { template <typename V> __device__ V operator()(V a, V b) const { return a + b; } };
struct Larger { __device__ float operator()(float a, float b) const { return __builtin_elementwise_maximum(a, b); } };     // NaN if one is

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
template <typename F>
hipError_t by_type(int type, F&& f) {
  switch (type) {
    case kF32: return f(float{});
    case kBF16: return f(bf16{});
    case kF16: return f(f16{});
    default: return hipErrorInvalidValue;
  }
}

// A launch has fewer than 2^32 threads: longer tensors go in slabs of samples.
template <typename F>
hipError_t by_slabs(int64_t samples, uint32_t pieces, F&& launch) {
  const int64_t slab = (int64_t(1) << 31) / pieces;
  for (int64_t at = 0; at < samples; at += slab) {
    const int64_t n = std::min(slab, samples - at);
    hipError_t e = launch(at, n, (unsigned)((n * pieces + 255) / 256));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// a tile's end
// ---------------------------------------------------------------------------
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x8 lds_s16x8;

// How a tile's sums leave the matrix instructions' layout: a wavefront's blocks of FI x FJ go to LDS strip by strip, 32 rows j of
// 32 FI values, and come back with the lanes along the rows, N values of i each, so that each instruction that stores them writes
// whole runs of memory (16 bytes a lane scattered over 64 rows took four times as long).  Pieces of 64 lanes are numbered through the tile.
// Chunks of 4 values change places within a row as a tile's do, for writes of one chunk of 32 rows and reads along rows.
template <int FI, int FJ, int WI, int WJ, int N>
struct Strips {
  static constexpr int lanes = FI * 32 / N, rows = 64 / lanes, turns = 32 / rows, chunks = FI * 8, bytes = 32 * chunks * 16;
  static constexpr int per_wave = FJ * turns, pieces = WI * WJ * per_wave;
  __device__ static inline int column(int piece, int lane) { return piece / per_wave % WI * (FI * 32) + lane % lanes * N; }
  __device__ static inline int row(int piece, int lane) {
    return (piece / per_wave / WI * FJ + piece / turns % FJ) * 32 + piece % turns * rows + lane / lanes;
  }
  // A lane that takes two chunks back finds the even ones in the first half of a row and the odd ones in the second: neighbouring
  // lanes read neighbouring places.
  __device__ static inline int place(int row, int chunk) {
    const int at = N == 4 ? chunk : (chunk >> 1) + (chunk & 1) * (chunks / 2);
    return (row * chunks + (at ^ (row & (chunks - 1)))) * 16;
  }
  __device__ static inline void put(lds_char* strip, int k, const f32x16& block, int lane) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float x[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = block[4 * g + c];
      s16x8 v;
      __builtin_memcpy(&v, x, 16);
      *reinterpret_cast<lds_s16x8*>(strip + place(lane & 31, 8 * k + 2 * g + (lane >> 5))) = v;
    }
  }
  // What piece `turn` of a strip has for a lane.
  __device__ static inline void get(float (&v)[N], const lds_char* strip, int turn, int lane) {
    const int row = turn * rows + lane / lanes, u = lane % lanes;
    if constexpr (N == 4) {
      const s16x8 x = *reinterpret_cast<const lds_s16x8*>(strip + place(row, u));
      __builtin_memcpy(v, &x, 16);
    } else {
      const s16x8 x = *reinterpret_cast<const lds_s16x8*>(strip + place(row, 2 * u)), y = *reinterpret_cast<const lds_s16x8*>(strip + place(row, 2 * u + 1));
      __builtin_memcpy(v, &x, 16);
      __builtin_memcpy(v + 4, &y, 16);
    }
  }
};

}  // namespace
}  // namespace linear
}  // namespace lqsgd
