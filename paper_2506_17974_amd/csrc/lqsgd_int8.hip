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

// A tile of N operand rows x K bytes, in chunks of 16, LDS rows end to end.  Chunks change places within a row so that the 32 rows that
// one instruction reads a chunk of lie in different banks.
template <int N, int K>
struct Tile {
  static constexpr int row_chunks = K / 16, chunks = row_chunks * N, bytes = chunks * 16;
  __device__ static inline int moved(int row) {
    static_assert(row_chunks == 4 || row_chunks == 8, "the exchange stays within a row");
    return row_chunks == 8 ? (row & 7) ^ (row >> 3 & 1) : (row >> 1 & 3) ^ (row >> 3 & 1);
  }
  __device__ static inline int place(int row, int chunk) { return (row * row_chunks + (chunk ^ moved(row))) * 16; }
  // The 16 codes that a lane holds of rows n0 .. n0 + 31 and r = r0 .. r0 + 31 (n0, r0 multiples of 32).
  __device__ static inline i32x4 fragment(const lds_char* tile, int n0, int r0, int lane) {
    return *reinterpret_cast<const lds_i32x4*>(tile + place(n0 + (lane & 31), r0 / 16 + (lane >> 5)));
  }
};

// One operand of a workgroup's tile and its way into LDS: 16 bytes a lane, straight from memory.  Lanes that have nothing there get an
// offset out of the buffer's range, which reads as 0.  The load is written out because the compiler, which knows what it writes but
// not which of it has been waited for, would wait for all of them before any read of LDS: whoever calls this waits for it (vmcnt)
// before a barrier and the first read.
template <int N, int K, int THREADS>
struct Operand {
  using L = Tile<N, K>;
  static constexpr int loads = L::chunks / THREADS;
  static_assert(L::chunks % THREADS == 0, "the tile has to be shared out evenly");
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
      const int piece = (wave * loads + k) * 64 + lane, row = piece / L::row_chunks;
      offset[k] = row < n ? row * stride + (piece % L::row_chunks ^ L::moved(row)) * 16 : kNowhere;
    }
  }
  __device__ inline void load(lds_char* to, int r0, int last) const {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const uint64_t from = (uint64_t)(base + r0);
    const u32x4 buffer = {(uint32_t)from, (uint32_t)(from >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
    const uint32_t at = (uint32_t)(uintptr_t)to + (uint32_t)(wave * loads) * 1024;
    const int left = last - r0;
#pragma unroll
    for (int k = 0; k < loads; ++k) {
      int o = offset[k];
      if (left < K) {
        const int piece = (wave * loads + k) * 64 + lane;
        o = (piece % L::row_chunks ^ L::moved(piece / L::row_chunks)) * 16 < left ? o : kNowhere;
      }
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :: "s"(at + k * 1024), "v"(o), "s"(buffer) : "memory", "m0");
    }
  }
};

// What a kernel's workgroups look like: BI x BJ of D, WI x WJ wavefronts, steps of BK values of r, BUFFERS of them in LDS.
template <int BI_, int BJ_, int WI_, int WJ_, int BK_, int BUFFERS_>
struct Shape {
  static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_, BK = BK_, buffers = BUFFERS_, threads = 64 * WI * WJ, FI = BI / WI / 32, FJ = BJ / WJ / 32;
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

// A tile of D to a workgroup, operands through LDS in steps of BK.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::threads >= 512 ? 2 : 1) void int8_product_kernel(Int8Args a, int tiles_i, int tiles_j) {
  using A = Operand<S::BI, S::BK, S::threads>;
  using B = Operand<S::BJ, S::BK, S::threads>;
  constexpr int kBytes = A::L::bytes + B::L::bytes;
  // an array each: what is on its way into one is not waited for where another is read
  __shared__ __attribute__((aligned(1024))) char lds0[kBytes];
  __shared__ __attribute__((aligned(1024))) char lds1[kBytes];
  __shared__ __attribute__((aligned(1024))) char lds2[S::buffers > 2 ? kBytes : 16];
  __shared__ __attribute__((aligned(1024))) char lds3[S::buffers > 3 ? kBytes : 16];
  auto buffer = [&](int k) { return k == 0 ? (lds_char*)lds0 : k == 1 ? (lds_char*)lds1 : k == 2 ? (lds_char*)lds2 : (lds_char*)lds3; };
  const Where at = where(tiles_i, tiles_j);
  const int i0 = at.ti * S::BI;
  const int64_t j0 = (int64_t)at.tj * S::BJ;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int wi = wave % S::WI * (S::FI * 32), wj = wave / S::WI * (S::FJ * 32);
  A oa;
  B ob;
  oa.prepare(a.a, i0, a.ni, a.stride, t);
  ob.prepare(a.b, j0, a.nj, a.stride, t);
  const int last = a.stride;
  auto fetch = [&](lds_char* to, int r) {
    oa.load(to, r, last);
    ob.load(to + A::L::bytes, r, last);
  };
  i32x16 acc[S::FI][S::FJ] = {};
  struct Fragments { i32x4 a[S::FI], b[S::FJ]; } now, next;
  auto read = [&](Fragments& f, const lds_char* from, int r) {
#pragma unroll
    for (int k = 0; k < S::FI; ++k) f.a[k] = A::L::fragment(from, wi + 32 * k, r, lane);
#pragma unroll
    for (int k = 0; k < S::FJ; ++k) f.b[k] = B::L::fragment(from + A::L::bytes, wj + 32 * k, r, lane);
  };
  auto multiply = [&](const Fragments& f) {
#pragma unroll
    for (int k = 0; k < S::FI; ++k)
#pragma unroll
      for (int q = 0; q < S::FJ; ++q) acc[k][q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.a[k], f.b[q], acc[k][q], 0, 0, 0);
  };
  // A step's last products run from registers, behind the barrier that makes the next step's operands everyone's, beside the reads of
  // those; its buffer is free from that barrier on and is filled for `buffers` steps ahead.  What may still be on its way at the
  // barrier: the fetches of the steps behind the next.
  constexpr int kOnTheWay = (S::buffers - 2) * (A::loads + B::loads);
  static_assert(kOnTheWay < 64);
  constexpr int kWait = 0x0070 | (kOnTheWay & 15) | (kOnTheWay >> 4) << 14;            // vmcnt(kOnTheWay), lgkmcnt(0)
  auto step = [&](lds_char* const here, lds_char* const there, int r) {
#pragma unroll
    for (int k = 32; k < S::BK; k += 32) {
      read(next, here, k);
      __builtin_amdgcn_sched_barrier(0);              // the reads go first, for the products to hide them
      multiply(now);
      now = next;
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWait);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(here, r + S::buffers * S::BK);
    read(next, there, 0);
    __builtin_amdgcn_sched_barrier(0);
    multiply(now);
    now = next;
  };
#pragma unroll
  for (int k = 0; k < S::buffers; ++k) fetch(buffer(k), k * S::BK);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  read(now, buffer(0), 0);
  for (int r = 0; r < last;) {
#pragma unroll
    for (int k = 0; k < S::buffers; ++k) {
      step(buffer(k), buffer((k + 1) % S::buffers), r);
      r += S::BK;
      if (r >= last) break;
    }
  }

  // The tile's end, one strip of blocks after the other, by code that is there once.
  constexpr int N = std::is_same_v<T, float> ? 4 : 8;
  using P = Strips<S::FI, S::FJ, S::WI, S::WJ, N>;
  constexpr int kEach = kBytes / P::bytes;              // wavefronts that a buffer holds the strips of
  static_assert(kEach > 0 && (S::WI * S::WJ + kEach - 1) / kEach <= S::buffers, "the strips have to fit the operands' buffers");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  lds_char* const strip = buffer(wave / kEach) + (wave % kEach) * P::bytes;
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
  const int64_t ti = (a.ni + S::BI - 1) / S::BI, tj = (a.nj + S::BJ - 1) / S::BJ;
  if (ti * tj * S::threads >= int64_t(1) << 32) return hipErrorInvalidValue;
  int8_product_kernel<T, S><<<dim3((unsigned)(ti * tj)), S::threads, 0, s>>>(a, (int)ti, (int)tj);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_product(int type, const Int8Args& a, hipStream_t s) {
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    if (a.nj >= 1024 && a.ni >= 1024) return run_product<T, Shape<256, 256, 2, 4, 64, 4>>(a, s);
    return run_product<T, Shape<128, 128, 2, 2, 64, 4>>(a, s);
  });
}

}  // namespace linear
}  // namespace lqsgd
