// gfx950 kernels of the linear layer on 8-bit rows.
//
// Sums of products are exact 32-bit integers: the same whatever their order.
#include "lqsgd_block_kernels.h"
#include "lqsgd_linear_device.h"

#include <algorithm>
#include <cstdint>
#include <type_traits>

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

// A part of an operand in LDS: N rows x 128 codes, in chunks of 16, rows end to end: whole lines of memory (with rows of 64 codes the
// requests to L2 were what bounded the largest products: 4096 x 11008 -> 4096 185 us).  Chunks change places within a row so that the 32
// rows that one instruction reads a chunk of lie in different banks.
constexpr int kDeep = 128, kRowChunks = kDeep / 16;
__device__ inline int moved(int row) { return (row & 7) ^ (row >> 3 & 1); }
__device__ inline int place(int row, int chunk) { return (row * kRowChunks + (chunk ^ moved(row))) * 16; }

// One operand of a workgroup's tile and its way into LDS: 16 bytes a lane, straight from memory.  Lanes that have nothing there get an
// offset out of the buffer's range, which reads as 0.  The load is written out because the compiler, which knows what it writes but
// not which of it has been waited for, would wait for all of them before any read of LDS: whoever calls this waits for it (vmcnt)
// before a barrier and the first read.
template <int N, int THREADS>
struct Operand {
  static constexpr int loads = N * kRowChunks / THREADS;
  static_assert(N * kRowChunks % THREADS == 0, "the tile has to be shared out evenly");
  static constexpr int kNowhere = (int)0x80000000u;
  const int8_t* base;
  int offset[loads];
  int wave, lane;

  __device__ inline void prepare(const int8_t* from, int64_t row0, int64_t rows, int stride, int t) {
    base = from + row0 * stride;
    wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    const int n = (int)min((int64_t)N, rows - row0);
#pragma unroll
    for (int k = 0; k < loads; ++k) {
      const int piece = (wave * loads + k) * 64 + lane, row = piece / kRowChunks;
      offset[k] = row < n ? row * stride + (piece % kRowChunks ^ moved(row)) * 16 : kNowhere;
    }
  }
  // Piece k of `loads` of the part from r0 on.
  __device__ inline void load(int k, uint32_t to, int r0, int last) const {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const uint64_t from = (uint64_t)(base + r0);
    const u32x4 buffer = {(uint32_t)from, (uint32_t)(from >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
    int o = offset[k];
    if (last - r0 < kDeep) {
      const int piece = (wave * loads + k) * 64 + lane;
      o = (piece % kRowChunks ^ moved(piece / kRowChunks)) * 16 < last - r0 ? o : kNowhere;
    }
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(to + (uint32_t)(wave * loads + k) * 1024), "v"(o), "s"(buffer) : "memory", "m0");
  }
};

// What a kernel's workgroups look like: B_ x B_ of D, WI x WJ wavefronts.
template <int B_, int WI_, int WJ_>
struct Shape {
  static constexpr int B = B_, WI = WI_, WJ = WJ_, threads = 64 * WI * WJ, FI = B / WI / 32, FJ = B / WJ / 32, unit = B * kDeep, units = 5;
};

// The tile of a workgroup.  Workgroups go round the 8 XCDs; each XCD gets a run of consecutive tiles, which go in bands of 4 tile rows
// so that those that run together share operands in its L2.
struct Where { int ti, tj; };
__device__ inline Where where(int tiles_i, int tiles_j) {
  const int all = tiles_i * tiles_j, b = (int)blockIdx.x, x = b & 7, q = all >> 3, rem = all & 7;
  const int tile = x * q + min(x, rem) + (b >> 3);
  constexpr int kBand = 4;
  const int band = tile / (kBand * tiles_i), in = tile - band * kBand * tiles_i, high = min(kBand, tiles_j - band * kBand);
  return Where{in / high, band * kBand + in % high};
}

// A tile of D to a workgroup, operands through LDS in steps of 128 codes.  LDS holds five units, each a step of one operand: those of
// this step and the next, and the weight's of the step behind.  A step has four parts, whose products run from registers; the reads
// of the next part and the fetches are issued among them, one behind each product.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::threads >= 512 ? 2 : 1) void int8_product_kernel(Int8Args a, int tiles_i, int tiles_j) {
  using O = Operand<S::B, S::threads>;
  __shared__ __attribute__((aligned(1024))) char lds[S::units * S::unit];
  lds_char* const all = (lds_char*)lds;
  const Where at = where(tiles_i, tiles_j);
  const int i0 = at.ti * S::B;
  const int64_t j0 = (int64_t)at.tj * S::B;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), last = a.stride;
  O oa, ob;
  oa.prepare(a.a, i0, a.ni, a.stride, t);
  ob.prepare(a.b, j0, a.nj, a.stride, t);
  const uint32_t start = (uint32_t)(uintptr_t)all;
  // rows of the tile that this wavefront multiplies, as bytes of a unit, and where in it a lane finds its chunks of the four parts
  const int wi = wave % S::WI * (S::FI * 32) * kDeep, wj = wave / S::WI * (S::FJ * 32) * kDeep;
  int mine[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) mine[k] = place(lane & 31, 2 * k + (lane >> 5));

  i32x16 acc[S::FI][S::FJ] = {};
  struct Fragments { i32x4 a[S::FI], b[S::FJ]; } now, next;
  constexpr int kReads = S::FI + S::FJ, kProducts = S::FI * S::FJ;
  auto read = [&](Fragments& f, int k, int part, int ua, int ub) {
    if (k < S::FI) f.a[k] = *reinterpret_cast<const lds_i32x4*>(all + (ua + wi + mine[part] + k * 32 * kDeep));
    else f.b[k - S::FI] = *reinterpret_cast<const lds_i32x4*>(all + (ub + wj + mine[part] + (k - S::FI) * 32 * kDeep));
  };
  // The products from registers; among them the reads of the next operands, part `part` of the units at ua and ub, and loads
  // `from`-th to `to`-th of operand o's step at r into the unit at uo.
  auto multiply = [&](int part, int ua, int ub, const O& o, int from, int to, int uo, int r) {
#pragma unroll
    for (int k = 0; k < kProducts; ++k) {
      acc[k / S::FJ][k % S::FJ] = __builtin_amdgcn_mfma_i32_32x32x32_i8(now.a[k / S::FJ], now.b[k % S::FJ], acc[k / S::FJ][k % S::FJ], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = k * kReads / kProducts; q < (k + 1) * kReads / kProducts; ++q) read(next, q, part, ua, ub);
#pragma unroll
      for (int q = from + k * (to - from) / kProducts; q < from + (k + 1) * (to - from) / kProducts; ++q) o.load(q, start + uo, r, last);
      __builtin_amdgcn_sched_barrier(0);
    }
    now = next;
  };
  // Units go round: the weight's and the input's steps take every other one.
  auto behind = [](int u, int n) { u += n * S::unit; return u >= S::units * S::unit ? u - S::units * S::unit : u; };
#pragma unroll
  for (int k = 0; k < O::loads; ++k) {
    oa.load(k, start, 0, last);
    ob.load(k, start + S::unit, 0, last);
    oa.load(k, start + 2 * S::unit, kDeep, last);
    ob.load(k, start + 3 * S::unit, kDeep, last);
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kReads; ++k) read(now, k, 0, 0, S::unit);
  int ua = 0;
  for (int r = 0; r < last; r += kDeep) {
    const int ub = behind(ua, 1), next_a = behind(ua, 2), next_b = behind(ua, 3), third = behind(ua, 4);
    multiply(1, ua, ub, oa, 0, O::loads / 2, third, r + 2 * kDeep);
    multiply(2, ua, ub, oa, O::loads / 2, O::loads, third, r + 2 * kDeep);
    multiply(3, ua, ub, oa, 0, 0, 0, 0);
    // The next step's units have come (what may still be on its way: the weight's behind that), and nobody reads this step's any more.
    constexpr int kWait = 0x0070 | (O::loads & 15) | (O::loads >> 4) << 14;            // vmcnt(loads), lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWait);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    multiply(0, next_a, next_b, ob, 0, O::loads, ua, r + 2 * kDeep);
    ua = next_a;
  }

  // The tile's end, one strip of blocks after the other, by code that is there once.
  constexpr int N = std::is_same_v<T, float> ? 4 : 8;
  using P = Strips<S::FI, S::FJ, S::WI, S::WJ, N>;
  static_assert(S::WI * S::WJ * P::bytes <= S::units * S::unit, "the strips have to fit the operands' place");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  lds_char* const strip = all + wave * P::bytes;
#pragma clang loop unroll(disable)
  for (int q = 0; q < S::FJ; ++q) {
#pragma unroll
    for (int qq = 0; qq < S::FJ; ++qq) {
      if (qq != q) continue;
#pragma unroll
      for (int k = 0; k < S::FI; ++k) P::put(strip, k, __builtin_bit_cast(f32x16, acc[k][qq]), lane);
    }
#pragma clang loop unroll(disable)
    for (int turn = 0; turn < P::turns; ++turn) {
      const int piece = wave * P::per_wave + q * P::turns + turn;
      float v[N];
      int sum[N];
      P::get(v, strip, turn, lane);
      __builtin_memcpy(sum, v, sizeof v);
      finish<T>(sum, a, j0 + P::row(piece, lane), i0 + P::column(piece, lane));
    }
  }
}

template <typename T, typename S>
hipError_t run_product(const Int8Args& a, hipStream_t s) {
  const int64_t ti = (a.ni + S::B - 1) / S::B, tj = (a.nj + S::B - 1) / S::B;
  if (ti * tj * S::threads >= int64_t(1) << 32) return hipErrorInvalidValue;
  int8_product_kernel<T, S><<<dim3((unsigned)(ti * tj)), S::threads, 0, s>>>(a, (int)ti, (int)tj);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_product(int type, const Int8Args& a, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    if (a.nj >= 1024 && a.ni >= 1024) return run_product<T, Shape<256, 2, 4>>(a, s);
    return run_product<T, Shape<128, 2, 2>>(a, s);
  });
}

}  // namespace linear
}  // namespace lqsgd
