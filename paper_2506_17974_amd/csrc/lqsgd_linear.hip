// gfx950 kernels of the linear layer whose gradients the compressor takes: the three products of a layer (forward with its
// epilogue, input gradient, weight gradient from an 8-bit checkpoint), checkpoints, and the activation's backward pass.
//
// Sums have a fixed order: results are bit-identical run to run.
#include "lqsgd_linear_device.h"
#include "lqsgd_linear_kernels.h"
#include "lqsgd_linear_plan.h"

#include <algorithm>
#include <cstdint>
#include <type_traits>

namespace lqsgd {
namespace linear {
namespace {

// ---------------------------------------------------------------------------
// checkpoints
// ---------------------------------------------------------------------------
// A thread takes a piece of 8 consecutive values, four lanes a group; a workgroup a run of 256 pieces of the whole tensor, rows end to
// end, so that narrow tensors fill their lanes too.  Bound by memory: s + 33/32 bytes per value (four pieces a thread on their way at
// once: no faster, small tensors 2.8 -> 3.9 us).  8192 x 4096 bf16 values: saving 18 us (5.6 TB/s), loading 16 (6.2).
template <typename T>
__global__ __launch_bounds__(256) void checkpoint_save_kernel(const T* x, int64_t ldx, Codes c, int64_t samples, int features, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  const bool there = row < samples;
  float v[kPiece];
  load_values(v, x + row * ldx + piece * kPiece, there ? features - (int)(piece * kPiece) : 0);
  uint32_t w[2], byte;
  pack_codes<T>(w, v, group_largest<kPiece>(largest(v)), &byte);
  if (!there) return;
  *reinterpret_cast<uint2*>(c.codes + row * ((int64_t)pieces * kPiece) + piece * kPiece) = make_uint2(w[0], w[1]);
  if ((piece & 3u) == 0) c.exponents[row * (pieces >> 2) + (piece >> 2)] = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(256) void checkpoint_load_kernel(T* x, int64_t ldx, Codes c, int64_t samples, int features, uint32_t pieces) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / pieces;
  const uint32_t at = (uint32_t)(first - row0 * pieces) + threadIdx.x, piece = at % pieces;
  const int64_t row = row0 + at / pieces;
  if (row >= samples) return;
  const uint2 w = *reinterpret_cast<const uint2*>(c.codes + row * ((int64_t)pieces * kPiece) + piece * kPiece);
  float v[kPiece];
  decode(v, w, factor_of(c.exponents[row * (pieces >> 2) + (piece >> 2)]));
  store_values(x + row * ldx + piece * kPiece, v, features - (int)(piece * kPiece));
}

// ---------------------------------------------------------------------------
// activation backward
// ---------------------------------------------------------------------------
// Slopes as a table: z = |q| 2^e has 128 values an exponent, and act'(z) = 1 - act'(-z) for gelu and silu.  Entries are act'(-|z|), so
// that the slopes that go to 0 are held to a float's relative precision, as the formula has them.  Rows e = -32 (below, z is under 2^-25
// and the slope 1/2 to half a unit in its last place) to 7 (above, the slope is 0 or 1 for every |q| >= 1).
constexpr int kSlopes = kSlopeRows * 128, kSlopeLow = -32;
static_assert(kTiles <= kSlopeFloats && kSlopeFloats % 256 == 0);

// What a context's memory has to hold before its first call: the slopes, and no part of any tile's sum.
__global__ __launch_bounds__(256) void prepare_kernel(float* table, int* arrived) {
  const int at = (int)blockIdx.x * 256 + threadIdx.x;              // gelu's, then silu's
  if (at < kTiles) arrived[at] = 0;
  const int act = at < kSlopes ? kGelu : kSilu, in = at % kSlopes;
  const float z[1] = {-(float)(in & 127) * power_of_two(kSlopeLow + (in >> 7))};
  float d[1] = {1.f};
  times_slope(d, z, act);
  table[at] = d[0];
}

// d *= act'(z) of 8 codes of a group.
__device__ inline void times_tabled_slope(float (&d)[8], uint2 w, uint32_t byte, const float* table) {
  const float* row = table + min(max((int)byte - 127 - kSlopeLow, 0), kSlopeRows - 1) * 128;
  const float zero = byte == 255u ? __builtin_nanf("") : 0.f, one = byte == 255u ? __builtin_nanf("") : 1.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int q = (int8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
    const float t = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, row[abs(q) & 127]) ^ (~(uint32_t)q & 0x80000000u));
    d[k] *= (q < 0 ? zero : one) + t;
  }
}

// A workgroup takes a strip of 8 << lanes_log2 features and a run of samples; a lane keeps 8 features' sums and has 4 samples on
// their way.  Lanes that the strip does not fill take further samples.  Strips' sums over runs go to `part` (runs x rows) where
// there is more than one run.  TABLE: gelu or silu of many samples, slopes from LDS (by formulas of 27 instructions a value the
// vector units took 54 us for 4096 x 11008 bfloat16 values; now 42, and 58.6 a pass where the tensors come from HBM: 3.9 TB/s, where plain
// streams of this mix reach 6.2 -- pieces of 1 KiB lie 22 KB apart, and 60 % of the table reads' LDS cycles are bank conflicts).
template <typename T, bool TABLE>
__global__ __launch_bounds__(256) void activation_backward_kernel(const T* dy, int64_t lddy, Codes z, T* dz, int64_t lddz, float* dbias,
                                                                  int accumulate, float* part, const float* slopes, int64_t samples,
                                                                  int rows, int act, int lanes_log2, int64_t run) {
  __shared__ float sums[256][kPiece + 1];
  __shared__ float table[TABLE ? kSlopes : 1];
  const int lanes = 1 << lanes_log2, t = threadIdx.x;
  if constexpr (TABLE) {
    for (int k = t * 4; k < kSlopes; k += 1024) *reinterpret_cast<float4*>(table + k) = *reinterpret_cast<const float4*>(slopes + k);
    __syncthreads();
  }
  const int feature = ((int)blockIdx.x * lanes + (t & (lanes - 1))) * kPiece;
  const int n = rows - feature;
  const int groups = (rows + kGroup - 1) / kGroup;
  const int64_t first = (int64_t)blockIdx.y * run, last = min(samples, first + run);
  float s[kPiece] = {};
  if (n > 0) {
    constexpr int kAtOnce = 4;
    const int step = 256 >> lanes_log2;
    for (int64_t m = first + (t >> lanes_log2); m < last; m += kAtOnce * step) {
      float v[kAtOnce][kPiece];
      uint2 w[kAtOnce] = {};
      uint32_t e[kAtOnce] = {};
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int64_t row = min(m + k * step, last - 1);   // beyond the end: read, not used
        load_values(v[k], dy + row * lddy + feature, n);
        if (act == kNone) continue;
        w[k] = *reinterpret_cast<const uint2*>(z.codes + row * ((int64_t)groups * kGroup) + feature);
        e[k] = z.exponents[row * groups + feature / kGroup];
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int64_t row = m + k * step;
        if (row >= last) break;
        if constexpr (TABLE) {
          times_tabled_slope(v[k], w[k], e[k], table);
        } else if (act != kNone) {
          float zv[kPiece];
          decode(zv, w[k], factor_of(e[k]));
          times_slope(v[k], zv, act);
        }
        if (dz) store_values(dz + row * lddz + feature, v[k], n);
#pragma unroll
        for (int c = 0; c < kPiece; ++c) s[c] += v[k][c];
      }
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

// Features' sums over `runs` runs of samples, in the runs' order by four.
__global__ __launch_bounds__(256) void sum_runs_kernel(const float* part, float* dbias, int accumulate, int rows, int runs) {
  __shared__ float sums[4][64];
  const int f = (int)blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float s = 0.f;
  if (f < rows) {
#pragma unroll 8
    for (int k = w; k < runs; k += 4) s += part[(int64_t)k * rows + f];
  }
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
// 4096 x 11008 values with gelu and both checkpoints take 381 us with the product, 330 without all that: 50 vector instructions a
// value, whose time no product hides (a CU holds one 256 x 256 tile).
// The end of a product: v holds D[j][i0 .. i0 + N - 1], i0 a multiple of N, and neighbouring lanes the rest of the group of 32.  All
// lanes of the wavefront come here together; `there` is false for those that have no row j.  N: 16 bytes of what is written.
template <typename T, int PRODUCT> constexpr int kRun = std::is_same_v<T, float> || PRODUCT == kWeightGrad ? 4 : 8;

template <typename T, int PRODUCT, int N>
__device__ inline void load_bias(float (&b)[N], const ProductArgs& a, int i0) {
  if (PRODUCT != kForward) return;
  load_values(b, static_cast<const T*>(a.bias) + i0, a.bias ? a.ni - i0 : 0);
}

template <typename T, int PRODUCT, int N>
__device__ inline void finish(float (&v)[N], const float (&bias)[N], const ProductArgs& a, int64_t j, int i0, bool there) {
  const int n = there ? a.ni - i0 : 0;
  if (PRODUCT == kWeightGrad) {
    if (n <= 0) return;
    if (a.out_type == kF32) {
      float* out = static_cast<float*>(a.out) + j * a.ldo + i0;
      if (a.accumulate) {
        float before[N];
        load_values(before, out, n);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += before[k];
      }
      store_values(out, v, n);
    } else {
      bf16* out = static_cast<bf16*>(a.out) + j * a.ldo + i0;
      if (a.accumulate) {
        float before[N];
        load_values(before, out, n);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += before[k];
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
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] += bias[k];
  auto keep = [&](const Codes& c) {
    if (n < N) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = k < n ? v[k] : 0.f;
    }
    uint32_t w[N / 4], byte;
    pack_codes<T>(w, v, group_largest<N>(largest(v)), &byte);
    if (in_codes) {
      __builtin_memcpy(__builtin_assume_aligned(c.codes + code_at, N), w, N);
      if (i0 % kGroup == 0) c.exponents[exp_at] = (uint8_t)byte;
    }
  };
  if (a.z.codes) keep(a.z);
  activate_all(v, a.act);
  if (a.residual) {
    float r[N];
    load_values(r, static_cast<const T*>(a.residual) + j * a.ldr + i0, n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += r[k];
  }
  if (n > 0) store_values(out, v, n);
  if (a.y.codes) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = widen(narrow<T>(v[k]));
    keep(a.y);
  }
}

// ---- operands: how a tile gets into LDS, and from there into the matrix instructions ----
// v_mfma_f32_32x32x16: a lane holds 8 consecutive r of operand row (lane mod 32), r0 = 8 (lane / 32); D comes back with
// i = 8 (v / 4) + 4 (lane / 32) + v mod 4 in register v, j = lane mod 32.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

template <typename E>
__device__ inline f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (std::is_same_v<E, f16>)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

enum Order {
  kDepthRuns = 0,      // memory rows are operand rows, r contiguous: LDS rows too
  kIndexRuns = 1,      // memory rows are values of r, operand rows contiguous: LDS rows hold one r, read through the transposing load
  kHeld = 2            // kIndexRuns from a checkpoint
};

// A tile of N operand rows x K values of r, 16-bit elements in chunks of 8 (16 bytes), LDS rows end to end.  Chunks change places
// within a row so that what one instruction reads lies in different banks, whether it is served 128 or 256 bytes at a time:
//   kDepthRuns: ds_read_b128 of one chunk of 32 rows;  kIndexRuns: ds_read_b64_tr_b16 of 4 values of r x 16 or 32 rows.
template <int ORDER, int N, int K>
struct Tile {
  static constexpr int row_chunks = ORDER == kDepthRuns ? K / 8 : N / 8;
  static constexpr int rows = ORDER == kDepthRuns ? N : K;
  static constexpr int chunks = row_chunks * rows;
  static constexpr int bytes = chunks * 16;
  __device__ static inline int moved(int row) {
    static_assert(row_chunks == 4 || row_chunks == 8 || (ORDER == kDepthRuns ? row_chunks == 2 : row_chunks % 16 == 0), "the exchange stays within a row");
    if (ORDER != kDepthRuns) {            // pairs of chunks
      if (row_chunks == 4) return row & 2;
      if (row_chunks == 8) return (row & 3) << 1;
      return (2 * (row & 1) + 5 * (row >> 1 & 1)) << 1;
    }
    return row_chunks == 8 ? (row & 7) ^ (row >> 3 & 1) : row_chunks == 4 ? (row >> 1 & 3) ^ (row >> 3 & 1) : (row >> 2 ^ row >> 3) & 1;
  }
  __device__ static inline int place(int row, int chunk) { return (row * row_chunks + (chunk ^ moved(row))) * 16; }
  // The 8 elements that a lane holds of rows n0 .. n0 + 31 and r = r0 .. r0 + 15 (n0 a multiple of 32, r0 of 16).
  __device__ static inline s16x8 fragment(const lds_char* tile, int n0, int r0, int lane) {
    if constexpr (ORDER == kDepthRuns) {
      return *reinterpret_cast<const lds_s16x8*>(tile + place(n0 + (lane & 31), r0 / 8 + (lane >> 5)));
    } else {
      // each 16 lanes read 4 values of r x 16 rows and get them back by rows
      const int r = r0 + 8 * (lane >> 5) + (lane >> 2 & 3), n = n0 + (lane & 16) + 4 * (lane & 3);
      lds_char* at = const_cast<lds_char*>(tile) + place(r, n / 8) + 2 * (n & 7);
      const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(at));
      const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(at + 4 * row_chunks * 16));
      return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

struct Chunk16 { uint32_t w[4]; };

// The first `valid` (0 .. 16 / sizeof(T)) elements from p, zeros behind them, without a branch and without touching memory beyond
// them: the 16 bytes that end there are read and shifted down.  There have to be 16 bytes of the tensor up to there; 16 bytes at `safe` are read
// where valid is 0.
template <typename T>
__device__ inline Chunk16 load_tail(const T* p, int valid, const T* safe) {
  constexpr int kAll = 16 / (int)sizeof(T);
  Chunk16 c;
  __builtin_memcpy(&c, valid > 0 ? p + (valid - kAll) : safe, 16);
  const int bytes = (kAll - valid) * (int)sizeof(T);
  const bool one = bytes & 4, two = bytes & 8;
  uint32_t w0 = one ? c.w[1] : c.w[0], w1 = one ? c.w[2] : c.w[1], w2 = one ? c.w[3] : c.w[2], w3 = one ? 0u : c.w[3];
  w0 = two ? w2 : w0, w1 = two ? w3 : w1, w2 = two ? 0u : w2, w3 = two ? 0u : w3;
  if (sizeof(T) == 2) {
    const uint32_t half = (bytes & 2) * 8;
    w0 = __builtin_amdgcn_alignbit(w1, w0, half), w1 = __builtin_amdgcn_alignbit(w2, w1, half);
    w2 = __builtin_amdgcn_alignbit(w3, w2, half), w3 = w3 >> half;
  }
  const uint32_t keep = valid > 0 ? 0xffffffffu : 0u;
  return Chunk16{{w0 & keep, w1 & keep, w2 & keep, w3 & keep}};
}

// fp32 in three bfloat16 terms, x = x1 + x2 + x3: the first cut off (so that it cannot overflow), the second rounded, the third exact.
__device__ inline void split3(const float (&x)[8], Chunk16 (&c)[3]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t h[2], m[2], l[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float v = x[2 * k + q];
      h[q] = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
      const float rest = v - __builtin_bit_cast(float, h[q]);
      const bf16 second = narrow<bf16>(rest);
      m[q] = __builtin_bit_cast(uint16_t, second);
      l[q] = __builtin_bit_cast(uint32_t, rest - widen(second)) >> 16;
    }
    c[0].w[k] = h[0] >> 16 | h[1];
    c[1].w[k] = m[0] | m[1] << 16;
    c[2].w[k] = l[0] | l[1] << 16;
  }
}

// One operand of a workgroup's tile: where it lies, and its way into LDS.  T: type in memory; E: element type in LDS; PLANES: 3 for
// fp32, else 1; THREADS of the workgroup.
template <typename T, typename E, int ORDER, int N, int K, int PLANES, int THREADS, bool DIRECT>
struct Operand {
  using L = Tile<ORDER, N, K>;
  static constexpr int bytes = L::bytes * PLANES;
  // kHeld: a thread takes 16 codes, two chunks.  Some wavefronts may have no part of a small tile.
  static constexpr int pieces = ORDER == kHeld ? L::chunks / 2 : L::chunks, per_thread = (pieces + THREADS - 1) / THREADS;
  static_assert(pieces % 64 == 0 && (!DIRECT || pieces % THREADS == 0), "the tile has to be shared out evenly");
  __device__ static inline bool mine(int piece) { return pieces % THREADS == 0 || piece < pieces; }

  const T* base;         // row n0 (kDepthRuns) or column n0 (kIndexRuns)
  int64_t ld;
  Codes held; int groups;
  int n;                 // operand rows from n0 on, N at most
  int length;            // of a memory row: the tensor's
  int64_t depth;
  int t;

  // in flight between load() and store()
  struct Empty {};
  using Raw = std::conditional_t<std::is_same_v<T, float>, float[8], Chunk16>;
  struct Regs {
    std::conditional_t<DIRECT || ORDER == kHeld, Empty, Raw[per_thread]> raw;
    std::conditional_t<ORDER == kHeld, Chunk16[per_thread], Empty> codes;
    std::conditional_t<ORDER == kHeld, uint32_t[per_thread], Empty> exps;
    std::conditional_t<ORDER == kHeld, bool[per_thread], Empty> there;
  };

  // Straight into LDS, 16 bytes a lane: memory rows start at multiples of 16 bytes and are whole chunks.  Lanes that have nothing
  // there get an offset out of the buffer's range, which reads as 0.  The load is written out because the compiler, which knows
  // what it writes but not which of it has been waited for, would wait for all of them before any read of LDS: whoever calls this
  // waits for it (vmcnt) before a barrier and the first read.
  static constexpr int kNowhere = (int)0x80000000u;
  int offset[DIRECT ? per_thread : 1];
  __device__ inline void prepare_direct() {
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
#pragma unroll
    for (int k = 0; k < per_thread; ++k) {
      const int piece = (wave * per_thread + k) * 64 + lane, row = piece / L::row_chunks;
      const int chunk = (piece % L::row_chunks) ^ L::moved(row);
      offset[k] = (ORDER == kDepthRuns ? row : chunk * 8) < n ? (row * (int)ld + chunk * 8) * 2 : kNowhere;
    }
  }
  __device__ inline void load_direct(lds_char* to, int64_t r0) const {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    const uint64_t from = (uint64_t)(base + (ORDER == kDepthRuns ? r0 : r0 * ld));
    const u32x4 buffer = {(uint32_t)from, (uint32_t)(from >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
    const uint32_t at = (uint32_t)(uintptr_t)to + (uint32_t)(wave * per_thread) * 1024;
    const int64_t left = depth - r0;
#pragma unroll
    for (int k = 0; k < per_thread; ++k) {
      int o = offset[k];
      if (left < K) {
        const int piece = (wave * per_thread + k) * 64 + lane, row = piece / L::row_chunks;
        const int r = ORDER == kDepthRuns ? ((piece % L::row_chunks) ^ L::moved(row)) * 8 : row;
        o = r < left ? o : kNowhere;
      }
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :: "s"(at + k * 1024), "v"(o), "s"(buffer) : "memory", "m0");
    }
  }

  // Through registers: memory of any alignment, rows of any length.
  __device__ inline void load(Regs& g, int64_t r0) {
    const int left = (int)min((int64_t)K, depth - r0);
    if constexpr (ORDER == kHeld) {
#pragma unroll
      for (int k = 0; k < per_thread; ++k) {
        // loaded in any case, as product_kernel counts loads; codes go on to the end of their group of 32
        const int piece = k * THREADS + t, r = piece / (N / 16), i = piece % (N / 16) * 16;
        const int whole = (n + kGroup - 1) / kGroup * kGroup;
        const int64_t row = min(r0 + r, depth - 1);
        const int col = min(i, whole - 16);
        g.codes[k] = *reinterpret_cast<const Chunk16*>(held.codes + row * ((int64_t)groups * kGroup) + col);
        g.exps[k] = held.exponents[row * groups + col / kGroup];
        g.there[k] = r0 + r < depth && i < n;            // else zeros: decided when they have come
      }
    } else {
      const T* from = base + (ORDER == kDepthRuns ? r0 : r0 * ld);
      const int rows = ORDER == kDepthRuns ? n : left, run = ORDER == kDepthRuns ? left : n;
      constexpr int kPart = 16 / (int)sizeof(T), kParts = 8 / kPart;
      if (n == N && left == K) {
#pragma unroll
        for (int k = 0; k < per_thread; ++k) {
          const int piece = k * THREADS + t;
          if (!mine(piece)) break;
          __builtin_memcpy(&g.raw[k], from + (int64_t)(piece / L::row_chunks) * ld + piece % L::row_chunks * 8, 8 * sizeof(T));
        }
      } else if (length >= kPart) {
        const T* safe = from + (min(run, kPart) - kPart);      // a run that starts the tensor's first row is that long
#pragma unroll
        for (int k = 0; k < per_thread; ++k) {
          const int piece = k * THREADS + t, row = piece / L::row_chunks, chunk = piece % L::row_chunks;
          if (!mine(piece)) break;
#pragma unroll
          for (int h = 0; h < kParts; ++h) {
            const int valid = row < rows ? min(max(run - chunk * 8 - h * kPart, 0), kPart) : 0;
            const Chunk16 c = load_tail(from + (int64_t)row * ld + chunk * 8 + h * kPart, valid, safe);
            __builtin_memcpy(reinterpret_cast<char*>(&g.raw[k]) + 16 * h, &c, 16);
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < per_thread; ++k) {
          const int piece = k * THREADS + t, row = piece / L::row_chunks, chunk = piece % L::row_chunks;
          if (!mine(piece)) break;
          const T* p = from + (int64_t)row * ld + chunk * 8;
          T v[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = row < rows && q < run - chunk * 8 ? p[q] : T(0.f);
          __builtin_memcpy(&g.raw[k], v, 8 * sizeof(T));
        }
      }
    }
  }
  __device__ inline void store(const Regs& g, lds_char* to) const {
    if constexpr (ORDER == kHeld) {
#pragma unroll
      for (int k = 0; k < per_thread; ++k) {
        const int piece = k * THREADS + t, r = piece / (N / 16), i = piece % (N / 16) * 16;
        if (!mine(piece)) break;
        const float f = g.there[k] ? factor_of(g.exps[k]) : 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          E e[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) e[q] = narrow<E>((float)(int8_t)(g.codes[k].w[2 * h + q / 4] >> (8 * (q & 3))) * f);
          put(to + L::place(r, i / 8 + h), __builtin_bit_cast(Chunk16, e));
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < per_thread; ++k) {
        const int piece = k * THREADS + t, at = L::place(piece / L::row_chunks, piece % L::row_chunks);
        if (!mine(piece)) break;
        if constexpr (PLANES == 3) {
          Chunk16 c[3];
          split3(g.raw[k], c);
#pragma unroll
          for (int p = 0; p < 3; ++p) put(to + p * L::bytes + at, c[p]);
        } else {
          put(to + at, g.raw[k]);
        }
      }
    }
  }
  __device__ static inline void put(lds_char* to, const Chunk16& c) { *reinterpret_cast<lds_s16x8*>(to) = __builtin_bit_cast(s16x8, c); }
};

// What a kernel's workgroups look like: BI x BJ of D, WI x WJ wavefronts, steps of BK values of r, BUFFERS of them in LDS.
template <int BI_, int BJ_, int WI_, int WJ_, int BK_, int BUFFERS_>
struct Shape {
  static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_, BK = BK_, buffers = BUFFERS_, threads = 64 * WI * WJ, FI = BI / WI / 32, FJ = BJ / WJ / 32;
};

// The tile and split of a workgroup.  Workgroups go round the 8 XCDs; each XCD gets a run of consecutive tiles, which go in bands
// of 4 tile rows so that those that run together share operands in its L2.
struct Where { int ti, tj, split; };
__device__ inline Where where(int tiles_i, int tiles_j, int tiles, int splits) {
  const int all = tiles * splits, b = (int)blockIdx.x, x = b & 7, q = all >> 3, rem = all & 7;
  const int w = x * q + min(x, rem) + (b >> 3);
  const int split = w / tiles, tile = w - split * tiles;
  constexpr int kBand = 4;
  const int band = tile / (kBand * tiles_i), in = tile - band * kBand * tiles_i, high = min(kBand, tiles_j - band * kBand);
  return Where{in / high, band * kBand + in % high, split};
}

// Types and operands of a product whose workgroups (or wavefronts: THREADS = 64) have a tile of BI x BJ, BK deep.
template <typename T, int PRODUCT, int BI, int BJ, int BK, int THREADS, bool DIRECT>
struct Operands {
  using E = std::conditional_t<std::is_same_v<T, f16>, f16, bf16>;
  static constexpr bool kWide = std::is_same_v<T, float>;
  static constexpr int kOrderA = PRODUCT == kForward ? kDepthRuns : PRODUCT == kInputGrad ? kIndexRuns : kHeld;
  static constexpr int kOrderB = PRODUCT == kWeightGrad ? kIndexRuns : kDepthRuns;
  static constexpr int PA = kWide && PRODUCT != kWeightGrad ? 3 : 1, PB = kWide ? 3 : 1;
  static constexpr bool kDirectA = DIRECT && kOrderA != kHeld;
  using A = Operand<T, E, kOrderA, BI, BK, PA, THREADS, kDirectA>;
  using B = Operand<T, E, kOrderB, BJ, BK, PB, THREADS, DIRECT>;
  static constexpr int bytes = A::bytes + B::bytes;
  A a;
  B b;

  __device__ inline Operands(const ProductArgs& p, int i0, int64_t j0, int64_t last, int t) {
    a.ld = p.lda; a.n = min(BI, p.ni - i0); a.depth = last; a.t = t;
    a.length = kOrderA == kDepthRuns ? (int)p.depth : p.ni;
    if constexpr (kOrderA == kHeld) {
      a.groups = (p.ni + kGroup - 1) / kGroup;
      a.held = Codes{p.held.codes + i0, p.held.exponents + i0 / kGroup};
    } else {
      a.base = static_cast<const T*>(p.a) + (kOrderA == kDepthRuns ? i0 * p.lda : i0);
    }
    b.ld = p.ldb; b.n = (int)min((int64_t)BJ, p.nj - j0); b.depth = last; b.t = t;
    b.length = kOrderB == kDepthRuns ? (int)p.depth : (int)p.nj;
    b.base = static_cast<const T*>(p.b) + (kOrderB == kDepthRuns ? j0 * p.ldb : j0);
    if constexpr (kDirectA) a.prepare_direct();
    if constexpr (DIRECT) b.prepare_direct();
  }
  static constexpr bool kRegisters = !kDirectA || !DIRECT;     // something goes through registers
  static constexpr int direct_loads = (kDirectA ? A::per_thread : 0) + (DIRECT ? B::per_thread : 0);
  static constexpr int held_loads = kOrderA == kHeld ? 2 * A::per_thread : 0;
  struct Regs {
    typename A::Regs a;
    typename B::Regs b;
  };
  // Values of r from r0 on: fetch() brings those that go straight into LDS (beyond the end: zeros), request() asks for those that
  // go through registers, deliver() puts those into LDS.
  __device__ inline void fetch(lds_char* to, int64_t r0) {
    if constexpr (kDirectA) a.load_direct(to, r0);
    if constexpr (DIRECT) b.load_direct(to + A::bytes, r0);
  }
  __device__ inline void request(Regs& g, int64_t r0) {
    if constexpr (!kDirectA) a.load(g.a, r0);
    if constexpr (!DIRECT) b.load(g.b, r0);
  }
  __device__ inline void deliver(const Regs& g, lds_char* to) const {
    if constexpr (!kDirectA) a.store(g.a, to);
    if constexpr (!DIRECT) b.store(g.b, to + A::bytes);
  }
  // The operands of 16 values of r, FI x FJ blocks from rows wi, wj of the tile on, and acc += their products.
  template <int FI, int FJ>
  struct Fragments {
    s16x8 a[PA][FI], b[PB][FJ];
    __device__ inline void read(const lds_char* from, int wi, int wj, int r, int lane) {
#pragma unroll
      for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int k = 0; k < FI; ++k) a[p][k] = A::L::fragment(from + p * A::L::bytes, wi + 32 * k, r, lane);
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int k = 0; k < FJ; ++k) b[p][k] = B::L::fragment(from + A::bytes + p * B::L::bytes, wj + 32 * k, r, lane);
    }
    __device__ inline void multiply(f32x16 (&acc)[FI][FJ]) const {
      // products of terms whose places add up to 2, 1, 0: the smaller ones first; those beyond are under 2^-22 of the product
#pragma unroll
      for (int sum = PA + PB > 2 ? 2 : 0; sum >= 0; --sum)
#pragma unroll
        for (int p = 0; p < PA; ++p) {
          if (sum - p < 0 || sum - p >= PB) continue;
#pragma unroll
          for (int k = 0; k < FI; ++k)
#pragma unroll
            for (int q = 0; q < FJ; ++q) acc[k][q] = mfma<E>(a[p][k], b[sum - p][q], acc[k][q]);
        }
    }
  };
};

// Where the sums of a piece of a split wait for the join: lanes side by side.
template <int N>
__device__ inline float* waiting(const ProductArgs& a, int64_t split, int64_t tile, int64_t tiles, int piece, int pieces, int lane) {
  return static_cast<float*>(a.workspace) + ((split * tiles + tile) * pieces + piece) * (64 * N) + lane * 4;
}
template <int N, bool ATOMIC>
__device__ inline void put_waiting(float* to, const float (&v)[N]) {
#pragma unroll
  for (int c = 0; c < N / 4; ++c) {
    if constexpr (ATOMIC) {
      uint64_t x[2];
      __builtin_memcpy(x, v + 4 * c, 16);
      uint64_t* p = reinterpret_cast<uint64_t*>(to + c * 256);
      __hip_atomic_store(p, x[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(p + 1, x[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
      *reinterpret_cast<float4*>(to + c * 256) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
    }
  }
}

template <int N, bool ATOMIC>
__device__ inline void add_parts(float (&v)[N], const ProductArgs& a, const Split& sp, int64_t tile, int piece, int pieces, int lane) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.f;
#pragma unroll 4
  for (int s = 0; s < sp.splits; ++s) {
    const float* from = waiting<N>(a, s, tile, (int64_t)sp.tiles_i * sp.tiles_j, piece, pieces, lane);
#pragma unroll
    for (int c = 0; c < N / 4; ++c) {
      float w[4];
      if constexpr (ATOMIC) {
        const uint64_t* p = reinterpret_cast<const uint64_t*>(from + c * 256);
        const uint64_t x[2] = {__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                               __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
        __builtin_memcpy(w, x, 16);
      } else {
        __builtin_memcpy(w, __builtin_assume_aligned(from + c * 256, 16), 16);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * c + e] += w[e];
    }
  }
}

// A tile of D to a workgroup, operands through LDS in steps of BK.  What bounds it: 32 x 32 x 16 matrix instructions at 1024 flops a
// cycle and SIMD, whose pipes are busy 47 (forward with its epilogue) to 65 % (input gradient) of the time, at 1.8 to 2.0 GHz, and what LDS
// has to deliver to them, which is why a wavefront has as large a part of the tile as its registers hold (128 x 64: 6 reads of 1 KiB
// to 8 products).  Measured, back to back, bfloat16 256 x 256: forward 4096 x 4096 -> 11008 338 us (1.09 PFLOP/s; the library's
// product 406), input gradient 4096 x 11008 -> 4096 290 us (1.27 PFLOP/s; library 261), weight gradient of 8192 samples, 4096 x 4096,
// decoding included, 265 us (1.04 PFLOP/s; library, from a decoded operand, 223).  fp32 256 x 128: input gradient 2048 x 8192 -> 8192
// 1.33 ms (206 TFLOP/s of fp32, 1.24 PFLOP/s of its six bfloat16 products; the fp32 matrix instructions reach 153 in the library).
// Tried: two buffers and a full wait at the barrier (input gradient 385 us), four wavefronts of 128 x 128 (the compiler spills 130
// registers: 1.3 ms), wavefront priorities around the products (310 against 296), fp32 in steps of 16 (1.6 ms).
template <typename T, int PRODUCT, typename S, bool DIRECT>
__global__ __launch_bounds__(S::threads, S::threads >= 512 ? 2 : 1) void product_kernel(ProductArgs a, Split sp) {
  using O = Operands<T, PRODUCT, S::BI, S::BJ, S::BK, S::threads, DIRECT>;
  // an array each: what is on its way into one is not waited for where another is read
  __shared__ __attribute__((aligned(1024))) char lds0[O::bytes];
  __shared__ __attribute__((aligned(1024))) char lds1[O::bytes];
  __shared__ __attribute__((aligned(1024))) char lds2[S::buffers > 2 ? O::bytes : 16];
  __shared__ __attribute__((aligned(1024))) char lds3[S::buffers > 3 ? O::bytes : 16];
  auto buffer = [&](int k) { return k == 0 ? (lds_char*)lds0 : k == 1 ? (lds_char*)lds1 : k == 2 ? (lds_char*)lds2 : (lds_char*)lds3; };

  const Where at = where(sp.tiles_i, sp.tiles_j, sp.tiles_i * sp.tiles_j, sp.splits);
  const int i0 = at.ti * S::BI;
  const int64_t j0 = (int64_t)at.tj * S::BJ;
  const int64_t first = at.split * sp.steps, last = min(a.depth, first + sp.steps);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int wi = wave % S::WI * (S::FI * 32), wj = wave / S::WI * (S::FJ * 32);
  O o(a, i0, j0, last, t);

  f32x16 acc[S::FI][S::FJ] = {};

  // A step's last products run from registers, behind the barrier that makes the next step's operands everyone's, beside the reads of
  // those; its buffer is free from that barrier on and is filled for `buffers` steps ahead.  What goes through registers is put to
  // LDS a step ahead, with vector instructions (splitting, decoding) that one half of the wavefronts (a SIMD has one of each half)
  // executes before its first products and the other half behind them, beside the other's matrix instructions; it has been asked for
  // one step before (fp32, whose steps are long) or two.
  // What may still be on its way at the barrier: the fetches of the steps behind the next, and the codes asked for since the next
  // step's fetches were.
  constexpr int kOnTheWay = DIRECT ? (S::buffers - 2) * O::direct_loads + (S::buffers - 1) * O::held_loads : 63;
  static_assert(kOnTheWay < 64);
  constexpr int kWait = 0x0070 | (kOnTheWay & 15) | (kOnTheWay >> 4) << 14;            // vmcnt(kOnTheWay), lgkmcnt(0)
  constexpr int kSets = std::is_same_v<T, float> ? 1 : 2;
  const bool early = wave < S::WI * S::WJ / 2;
  typename O::template Fragments<S::FI, S::FJ> now, next;
  typename O::Regs set[kSets];
  auto request = [&](typename O::Regs& g, int64_t r) {
    if (DIRECT || r < last) o.request(g, r);
  };
  auto step = [&](lds_char* const here, lds_char* const there, typename O::Regs& g, int64_t r) {
    auto bring = [&]() {
      if (!O::kRegisters || r + S::BK >= last) return;
      o.deliver(g, there);
      request(g, r + (1 + kSets) * S::BK);
    };
    if (early) bring();
#pragma unroll
    for (int k = 16; k < S::BK; k += 16) {
      next.read(here, wi, wj, k, lane);
      // the reads go first, for the products to hide them (registers for that are left where nothing else goes through them)
      if constexpr (!O::kRegisters) __builtin_amdgcn_sched_barrier(0);
      now.multiply(acc);
      now = next;
    }
    if (!early) bring();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWait);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    o.fetch(here, r + S::buffers * S::BK);
    next.read(there, wi, wj, 0, lane);
    if constexpr (!O::kRegisters) __builtin_amdgcn_sched_barrier(0);
    now.multiply(acc);
    now = next;
  };
  if (first < last) {
#pragma unroll
    for (int k = 0; k < kSets; ++k) request(set[k], first + k * S::BK);
#pragma unroll
    for (int k = 0; k < S::buffers; ++k) o.fetch(buffer(k), first + k * S::BK);
    o.deliver(set[0], buffer(0));
    request(set[0], first + kSets * S::BK);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    now.read(buffer(0), wi, wj, 0, lane);
    static_assert(S::buffers % kSets == 0);
    for (int64_t r = first; r < last;) {
#pragma unroll
      for (int k = 0; k < S::buffers; ++k) {
        step(buffer(k), buffer((k + 1) % S::buffers), set[(k + 1) % kSets], r);
        r += S::BK;
        if (r >= last) break;
      }
    }
  }

  // The tile's end, one strip of blocks after the other, by code that is there once.
  using P = Strips<S::FI, S::FJ, S::WI, S::WJ, kRun<T, PRODUCT>>;
  constexpr int N = kRun<T, PRODUCT>;
  constexpr int kEach = O::bytes / P::bytes;              // wavefronts that a buffer holds the strips of
  static_assert(kEach > 0 && (S::WI * S::WJ + kEach - 1) / kEach <= S::buffers, "the strips have to fit the operands' buffers");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  lds_char* const strip = buffer(wave / kEach) + (wave % kEach) * P::bytes;
  const int i = i0 + P::column(wave * P::per_wave, lane);
  float bias[N];
  load_bias<T, PRODUCT>(bias, a, i);
#pragma clang loop unroll(disable)
  for (int q = 0; q < S::FJ; ++q) {
#pragma unroll
    for (int qq = 0; qq < S::FJ; ++qq) {
      if (qq != q) continue;
#pragma unroll
      for (int k = 0; k < S::FI; ++k) P::put(strip, k, acc[k][qq], lane);
    }
#pragma clang loop unroll(disable)
    for (int turn = 0; turn < P::turns; ++turn) {
      const int piece = wave * P::per_wave + q * P::turns + turn;
      float v[N];
      P::get(v, strip, turn, lane);
      const int64_t j = j0 + P::row(piece, lane);
      if (sp.splits > 1) {
        put_waiting<N, false>(waiting<N>(a, at.split, (int64_t)at.tj * sp.tiles_i + at.ti, (int64_t)sp.tiles_i * sp.tiles_j, piece, P::pieces, lane), v);
      } else {
        finish<T, PRODUCT>(v, bias, a, j, i, j < a.nj);
      }
    }
  }
}

// The same for few tiles, down to single tokens: a workgroup's 8 wavefronts each have the whole tile and every 8th step of the sum, in
// LDS of their own, so that nothing waits for another wavefront before the end, where the sums are added up in LDS in the wavefronts'
// order.  Bound by the latency of a step (1.0 to 1.6 us for 8 x 64 values of r in 16-bit types, 1.7 for 8 x 16 in fp32, where
// splitting takes as long as multiplying) and, for single tokens, by the weights' stream: 4096 -> 11008 bf16 17 us, 5.3 TB/s, where a
// tile of 128 x 128 takes 40.  1024 x 1024 x 1024 bf16 8 us, fp32 21.  Two steps on their way, half as long each: 10 and 24 us.
template <typename T, int PRODUCT, int BI, int BJ, int BK, int WAVES, bool DIRECT>
__global__ __launch_bounds__(WAVES * 64) void product_by_depth_kernel(ProductArgs a, Split sp) {
  using O = Operands<T, PRODUCT, BI, BJ, BK, 64, DIRECT>;
  constexpr int FI = BI / 32, FJ = BJ / 32, N = kRun<T, PRODUCT>;
  using P = Strips<FI, FJ, 1, 1, N>;
  constexpr int kPlace = O::bytes > FJ * P::bytes ? O::bytes : FJ * P::bytes;       // of a wavefront: its operands, then its sums
  __shared__ __attribute__((aligned(1024))) char lds[WAVES * kPlace];
  const Where at = where(sp.tiles_i, sp.tiles_j, sp.tiles_i * sp.tiles_j, sp.splits);
  const int i0 = at.ti * BI;
  const int64_t j0 = (int64_t)at.tj * BJ;
  const int64_t first = at.split * sp.steps, last = min(a.depth, first + sp.steps);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  lds_char* const all = (lds_char*)lds;
  lds_char* const mine = all + wave * kPlace;
  O o(a, i0, j0, last, lane);
  f32x16 acc[FI][FJ] = {};
  typename O::Regs g;
  int64_t r = first + wave * BK;
  if (r < last) {
    o.fetch(mine, r);
    o.request(g, r);
  }
  while (r < last) {
    o.deliver(g, mine);
    // what this wavefront asked for is there
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t next = r + WAVES * BK;
    if (next < last) o.request(g, next);
#pragma unroll
    for (int k = 0; k < BK; k += 16) {
      typename O::template Fragments<FI, FJ> f;
      f.read(mine, 0, 0, k, lane);
      f.multiply(acc);
    }
    // every fragment has been read before LDS is written again
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (DIRECT && next < last) {
      __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0)
      o.fetch(mine, next);
    }
    r = next;
  }
#pragma unroll
  for (int q = 0; q < FJ; ++q)
#pragma unroll
    for (int k = 0; k < FI; ++k) P::put(mine + q * P::bytes, k, acc[k][q], lane);
  __syncthreads();
  for (int piece = wave; piece < P::pieces; piece += WAVES) {
    float v[N] = {}, bias[N];
    const int i = i0 + P::column(piece, lane);
    const int64_t j = j0 + P::row(piece, lane);
    load_bias<T, PRODUCT>(bias, a, i);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      float x[N];
      P::get(x, all + w * kPlace + piece / P::turns * P::bytes, piece % P::turns, lane);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] += x[e];
    }
    if (sp.splits > 1) {
      put_waiting<N, true>(waiting<N>(a, at.split, (int64_t)at.tj * sp.tiles_i + at.ti, (int64_t)sp.tiles_i * sp.tiles_j, piece, P::pieces, lane), v);
    } else {
      finish<T, PRODUCT>(v, bias, a, j, i, j < a.nj);
    }
  }
  if (sp.splits == 1) return;
  // The workgroup that comes last to a tile adds up its parts, in the parts' order, whichever it is.  Parts are stored and read with
  // agent-scope atomics, which go past the caches that the XCDs do not share: every store has arrived when vmcnt says so, and the
  // barrier puts all of the workgroup's before its count.  (A release at agent scope would write back the XCD's whole L2, 8 us.)
  const int tile = at.tj * sp.tiles_i + at.ti;
  int* const arrived = a.arrived + tile;
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __syncthreads();
  if (t == 0) {
    const bool last_one = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == sp.splits - 1;
    if (last_one) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);        // for the next launch
    *reinterpret_cast<volatile int*>(lds) = last_one;
  }
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(lds) == 0) return;
  for (int piece = wave; piece < P::pieces; piece += WAVES) {
    float v[N], bias[N];
    const int i = i0 + P::column(piece, lane);
    const int64_t j = j0 + P::row(piece, lane);
    load_bias<T, PRODUCT>(bias, a, i);
    add_parts<N, true>(v, a, sp, tile, piece, P::pieces, lane);
    finish<T, PRODUCT>(v, bias, a, j, i, j < a.nj);
  }
}

// Adds up the splits of a product in their order and ends it, a piece of a tile to a wavefront.
template <typename T, int PRODUCT, typename P, int BI, int BJ>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a, Split sp) {
  constexpr int N = kRun<T, PRODUCT>;
  const int lane = threadIdx.x & 63;
  const int64_t all = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), tile = all / P::pieces;
  const int piece = (int)(all - tile * P::pieces);
  const int i = (int)(tile % sp.tiles_i) * BI + P::column(piece, lane);
  const int64_t j = tile / sp.tiles_i * BJ + P::row(piece, lane);
  float v[N], bias[N];
  load_bias<T, PRODUCT>(bias, a, i);
  add_parts<N, false>(v, a, sp, tile, piece, P::pieces, lane);
  finish<T, PRODUCT>(v, bias, a, j, i, j < a.nj);
}

template <typename T, int PRODUCT, typename P, int BI, int BJ>
hipError_t join(const ProductArgs& a, const Plan& p, hipStream_t s) {
  static_assert(P::pieces % 4 == 0);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.sp.splits == 1) return e;
  join_kernel<T, PRODUCT, P, BI, BJ><<<dim3((unsigned)(p.tiles * P::pieces / 4)), 256, 0, s>>>(a, p.sp);
  return hipGetLastError();
}

template <typename T, int PRODUCT, typename S, bool DIRECT>
hipError_t run_product(const ProductArgs& a, const Plan& p, hipStream_t s) {
  product_kernel<T, PRODUCT, S, DIRECT><<<dim3((unsigned)(p.tiles * p.sp.splits)), S::threads, 0, s>>>(a, p.sp);
  return join<T, PRODUCT, Strips<S::FI, S::FJ, S::WI, S::WJ, kRun<T, PRODUCT>>, S::BI, S::BJ>(a, p, s);
}

template <typename T, int PRODUCT, int BI, int BJ, int BK, int WAVES, bool DIRECT>
hipError_t run_by_depth(const ProductArgs& a, const Plan& p, hipStream_t s) {
  product_by_depth_kernel<T, PRODUCT, BI, BJ, BK, WAVES, DIRECT><<<dim3((unsigned)(p.tiles * p.sp.splits)), WAVES * 64, 0, s>>>(a, p.sp);
  return hipGetLastError();
}

bool whole_chunks(const void* p, int64_t ld, int64_t length) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && length % 8 == 0;
}

template <typename T, int PRODUCT, bool DIRECT>
hipError_t by_size(const ProductArgs& a, hipStream_t s) {
  const Plan p = plan_product(PRODUCT, std::is_same_v<T, float>, DIRECT, a.ni, a.nj, a.depth);
  if (p.tiles == 0) return hipErrorInvalidValue;
  if constexpr (std::is_same_v<T, float>) {
    if (p.kernel == kLarge) return run_product<T, PRODUCT, Shape<256, 128, 4, 2, 32, 2>, DIRECT>(a, p, s);
    if (p.kernel == kMiddle) return run_product<T, PRODUCT, Shape<128, 128, 2, 2, 32, 2>, DIRECT>(a, p, s);
    if (a.nj <= 32) return run_by_depth<T, PRODUCT, 64, 32, 32, 8, DIRECT>(a, p, s);
    return run_by_depth<T, PRODUCT, 64, 64, 16, 8, DIRECT>(a, p, s);
  } else {
    // operands that go through registers leave none for 256 x 256
    if (p.kernel == kLarge) return run_product<T, PRODUCT, std::conditional_t<DIRECT, Shape<256, 256, 2, 4, 32, 4>, Shape<256, 128, 4, 2, 32, 4>>, DIRECT>(a, p, s);
    if (p.kernel == kMiddle) return run_product<T, PRODUCT, Shape<128, 128, 2, 2, 32, 4>, DIRECT>(a, p, s);
    if (a.nj <= 32) return run_by_depth<T, PRODUCT, 64, 32, 64, 8, DIRECT>(a, p, s);
    return run_by_depth<T, PRODUCT, 64, 64, 64, 8, DIRECT>(a, p, s);
  }
}

template <typename T, int PRODUCT>
hipError_t product(const ProductArgs& a, hipStream_t s) {
  if constexpr (!std::is_same_v<T, float>) {
    const bool direct = (PRODUCT == kWeightGrad || whole_chunks(a.a, a.lda, PRODUCT == kForward ? a.depth : a.ni)) &&
                        whole_chunks(a.b, a.ldb, PRODUCT == kWeightGrad ? a.nj : a.depth);
    if (direct) return by_size<T, PRODUCT, true>(a, s);
  }
  return by_size<T, PRODUCT, false>(a, s);
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
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    return by_slabs(samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      const Codes part{c.codes + at * pieces * kPiece, c.exponents + at * (pieces >> 2)};
      checkpoint_save_kernel<T><<<dim3(blocks), 256, 0, s>>>(static_cast<const T*>(x) + at * ldx, ldx, part, n, features, pieces);
      return hipGetLastError();
    });
  });
}

hipError_t launch_checkpoint_load(int type, int64_t samples, int32_t features, Codes c, void* x, int64_t ldx, hipStream_t s) {
  const uint32_t pieces = (uint32_t)((features + kGroup - 1) / kGroup * (kGroup / kPiece));
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    return by_slabs(samples, pieces, [&](int64_t at, int64_t n, unsigned blocks) {
      const Codes part{c.codes + at * pieces * kPiece, c.exponents + at * (pieces >> 2)};
      checkpoint_load_kernel<T><<<dim3(blocks), 256, 0, s>>>(static_cast<T*>(x) + at * ldx, ldx, part, n, features, pieces);
      return hipGetLastError();
    });
  });
}

hipError_t launch_prepare(float* slopes, int* arrived, hipStream_t s) {
  prepare_kernel<<<dim3(kSlopeFloats / 256), 256, 0, s>>>(slopes, arrived);
  return hipGetLastError();
}

hipError_t launch_activation_backward(int type, int act, int64_t samples, int32_t rows, const void* dy, int64_t lddy, Codes z, void* dz,
                                      int64_t lddz, float* dbias, int accumulate, void* workspace, const float* slopes, hipStream_t s) {
  const int pieces = (rows + kPiece - 1) / kPiece;
  // Few samples: strips of 128 features leave 16 samples to go on at a time, and one launch does (64 x 1024 fp32 6.8 us instead of 6.4 + 2.1).
  const bool one_run = samples <= 256;
  int lanes_log2 = 0;
  while ((1 << lanes_log2) < pieces && lanes_log2 < (one_run ? 4 : 6)) ++lanes_log2;
  const int strips = (pieces + (1 << lanes_log2) - 1) >> lanes_log2;
  const int64_t at_once = 4 * (256 >> lanes_log2);
  // otherwise up to 1280 workgroups, the five a CU that run together (4096 x 11008 bf16: 58 us, 768 66, 2048 65)
  const int64_t most = std::max<int64_t>(1, 1280 / strips);
  const int64_t rounds = (samples + at_once * most - 1) / (at_once * most);
  const int64_t run = one_run ? samples : rounds * at_once;
  const int64_t runs = samples == 0 ? 1 : (samples + run - 1) / run;
  float* part = dbias && runs > 1 ? static_cast<float*>(workspace) : nullptr;
  // the table pays from about 12 samples a lane on
  const bool table = (act == kGelu || act == kSilu) && !one_run && rounds >= 3;
  if (act == kSilu) slopes += kSlopes;
  hipError_t e = by_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto* kernel = table ? activation_backward_kernel<T, true> : activation_backward_kernel<T, false>;
    kernel<<<dim3((unsigned)strips, (unsigned)runs), 256, 0, s>>>(static_cast<const T*>(dy), lddy, z, static_cast<T*>(dz), lddz, dbias, accumulate,
                                                                  part, slopes, samples, rows, act, lanes_log2, run);
    return hipGetLastError();
  });
  if (e != hipSuccess || !part) return e;
  sum_runs_kernel<<<dim3((unsigned)((rows + 63) / 64)), 256, 0, s>>>(part, dbias, accumulate, rows, (int)runs);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace lqsgd
