// gfx950 kernels of the linear layer on 8-bit rows.
//
// Sums of products are exact 32-bit integers: the same whatever their order.
#include "lqsgd_block_kernels.h"
#include "lqsgd_int8_plan.h"
#include "lqsgd_linear_device.h"

#include <algorithm>
#include <cstdint>
#include <type_traits>

namespace lqsgd {
namespace linear {
namespace {

// v_mfma_i32_16x16x64_i8: a lane holds 16 consecutive r of operand row (lane mod 16), r0 = 16 (lane / 16); D comes back with
// i = 4 (lane / 16) + register, j = lane mod 16.  (32 x 32 x 32 does as much a cycle, but the card gives it less power's worth: on random codes
// 3.4 POPS in a loop of nothing else, this one 4.0.)
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;

// The end of a product for D[j][i0 .. i0 + N - 1]: what it reads, which few samples' kernels ask for before their sums, and what it does.
template <typename T, int N>
struct End {
  float scale[N], bias[N], residual[N], of_b;
  int n;
  __device__ inline void load(const Int8Args& a, int64_t j, int i0) {
    n = j < a.nj ? a.ni - i0 : 0;
    of_b = n > 0 ? a.scales_b[j] : 0.f;
    load_values(scale, a.scales_a + i0, n);
    load_values(bias, static_cast<const T*>(a.bias) + i0, a.bias ? n : 0);
    load_values(residual, static_cast<const T*>(a.residual) + j * a.ldr + i0, a.residual ? n : 0);
  }
  __device__ inline void finish(const int (&sum)[N], const Int8Args& a, int64_t j, int i0) const {
    if (n <= 0) return;
    float v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = fmaf((float)sum[k], of_b * scale[k], bias[k]);
    activate_all(v, a.act);
    if (a.residual) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += residual[k];
    }
    store_values(static_cast<T*>(a.out) + j * a.ldo + i0, v, n);
  }
};

// A part of an operand in LDS: N rows x 128 codes, in chunks of 16, rows end to end: whole lines of memory (with rows of 64 codes the
// requests to L2 were what bounded the largest products: 4096 x 11008 -> 4096 185 us).  Chunks change places within a row so that the
// 16 rows that one instruction reads a chunk of lie in different banks.
constexpr int kRowChunks = kDeep / 16;
__device__ inline int moved(int row) { return row >> 1 & 7; }
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
    if (__builtin_expect(last - r0 < kDeep, 0)) {
      const int piece = (wave * loads + k) * 64 + lane;
      o = (piece % kRowChunks ^ moved(piece / kRowChunks)) * 16 < last - r0 ? o : kNowhere;
    }
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(to + (uint32_t)(wave * loads + k) * 1024), "v"(o), "s"(buffer) : "memory", "m0");
  }
};

// What a kernel's workgroups look like: B_ x B_ of D, WI x WJ wavefronts, operands of AHEAD steps in LDS.
template <int B_, int WI_, int WJ_, int AHEAD>
struct Shape {
  static constexpr int B = B_, WI = WI_, WJ = WJ_, threads = 64 * WI * WJ, FI = B / WI / 16, FJ = B / WJ / 16;
  static constexpr int ahead = AHEAD, units = 2 * AHEAD + 1, unit = B * kDeep;
};

// The tile of a workgroup.  Workgroups go round the 8 XCDs; each XCD gets a run of consecutive tiles, which go in bands of 4 tile rows
// so that those that run together share operands in its L2.
struct Where { int ti, tj, split; };
__device__ inline Where where(int tiles_i, int tiles_j, int splits) {
  const int tiles = tiles_i * tiles_j, all = tiles * splits, b = (int)blockIdx.x, x = b & 7, q = all >> 3, rem = all & 7;
  const int w = x * q + min(x, rem) + (b >> 3), split = w / tiles, tile = w - split * tiles;
  constexpr int kBand = 4;
  const int band = tile / (kBand * tiles_i), in = tile - band * kBand * tiles_i, high = min(kBand, tiles_j - band * kBand);
  return Where{in / high, band * kBand + in % high, split};
}

// A tile of D to a workgroup, operands through LDS in steps of 128 codes.  LDS holds the units (a step of one operand each) of `ahead` steps
// and the weight's of the step behind them.  A step has two parts, whose products run from registers; the reads of the next part and
// the fetches are issued among them, a weight's fragment read again as soon as its products are.
// Bound by the matrix pipes, and those by the card's power: of 4096 x 11008 -> 4096's 231 thousand cycles a workgroup (247 with a residual) 176 are
// matrix work, 84 % of the loop's 210, on random codes and on zeros alike, and the clock follows the codes: 143 us on quantised normal values at 1.65 to
// 1.8 GHz (2.6 POPS; cards 130 to 158), 98 us on zeros at 2.25.  A tile's
// start and end are hidden by no other tile's products (one fits a CU).  8192 x 4096 -> 4096 110 to 116 us, 4096 x 4096 -> 11008 163 (688
// tiles in 2.7 rounds, paid as 3).  Tried: four wavefronts of 128 x 128 (their fragments go to scratch, slower), four for the 128 x 128 tile (slower).
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::threads >= 512 ? 2 : 1) void int8_product_kernel(Int8Args a, Split sp) {
  using O = Operand<S::B, S::threads>;
  __shared__ __attribute__((aligned(1024))) char lds[S::units * S::unit];
  lds_char* const all = (lds_char*)lds;
  const Where at = where(sp.tiles_i, sp.tiles_j, sp.splits);
  const int i0 = at.ti * S::B;
  const int64_t j0 = (int64_t)at.tj * S::B;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int first = at.split * (int)sp.steps, last = min(a.stride, first + (int)sp.steps);
  O oa, ob;
  oa.prepare(a.a, i0, a.ni, a.stride, t);
  ob.prepare(a.b, j0, a.nj, a.stride, t);
  const uint32_t start = (uint32_t)(uintptr_t)all;
  // rows of the tile that this wavefront multiplies, as bytes of a unit, and where in it a lane finds its chunks of the two parts
  const int wi = wave % S::WI * (S::FI * 16) * kDeep, wj = wave / S::WI * (S::FJ * 16) * kDeep;
  const int mine[2] = {place(lane & 15, lane >> 4), place(lane & 15, 4 + (lane >> 4))};

  // scales and bias of the tile's rows and columns, one a thread: for its end
  float of_a = 0.f, of_b = 0.f, of_bias = 0.f;
  if (t < S::B && i0 + t < a.ni) of_a = a.scales_a[i0 + t], of_bias = a.bias ? widen(static_cast<const T*>(a.bias)[i0 + t]) : 0.f;
  if (t < S::B && j0 + t < a.nj) of_b = a.scales_b[j0 + t];

  i32x4 acc[S::FI][S::FJ] = {}, fa[S::FI], fb[2][S::FJ];
  auto read_a = [&](int k, int part, int u) { fa[k] = *reinterpret_cast<const lds_i32x4*>(all + (u + wi + mine[part] + k * 16 * kDeep)); };
  auto read_b = [&](int k, int part, int u) { fb[part][k] = *reinterpret_cast<const lds_i32x4*>(all + (u + wj + mine[part] + k * 16 * kDeep)); };
  auto products = [&](int i, int part) {
#pragma unroll
    for (int k = 0; k < S::FJ; ++k) acc[i][k] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[part][k], acc[i][k], 0, 0, 0);
  };
  // Units go round: the weight's and the input's steps take every other one.
  auto behind = [](int u, int n) { u += n * S::unit; return u >= S::units * S::unit ? u - S::units * S::unit : u; };
#pragma unroll
  for (int d = 0; d < S::ahead; ++d)
#pragma unroll
    for (int k = 0; k < O::loads; ++k) {
      oa.load(k, start + 2 * d * S::unit, first + d * kDeep, last);
      ob.load(k, start + (2 * d + 1) * S::unit, first + d * kDeep, last);
    }
  auto wait = [](auto still) {
    constexpr int kStill = decltype(still)::value;         // fetches that may be on their way
    static_assert(kStill < 64);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (kStill & 15) | (kStill >> 4) << 14);            // vmcnt(kStill), lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  wait(std::integral_constant<int, O::loads * 2 * (S::ahead - 1)>{});
#pragma unroll
  for (int k = 0; k < S::FJ; ++k) read_b(k, 0, S::unit);
#pragma unroll
  for (int k = 0; k < S::FI; ++k) read_a(k, 0, 0);
  // The second part's first kHold + 1 fragments are multiplied before the barrier, while the part's last reads come back.
  constexpr int kHold = S::FI >= 8 ? 1 : 0;
  constexpr int kSoon = (2 * S::FJ + S::FI - 1) / S::FI;          // the input's fragments, which all products need, are read in the first half of a part
  int ua = 0;
  for (int r = first; r < last; r += kDeep) {
    const int ub = behind(ua, 1), next_a = behind(ua, 2), next_b = behind(ua, 3), free = behind(ua, S::units - 1), ahead = r + S::ahead * kDeep;
#pragma unroll
    for (int i = 0; i < S::FI; ++i) {
      products(i, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = i * kSoon; k < std::min((i + 1) * kSoon, S::FJ); ++k) read_b(k, 1, ub);
      read_a(i, 1, ua);
#pragma unroll
      for (int k = i * O::loads / S::FI; k < (i + 1) * O::loads / S::FI; ++k) oa.load(k, start + free, ahead, last);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < S::FI; ++i) {
      products(i, 1);
      __builtin_amdgcn_sched_barrier(0);
      if (i < kHold) continue;
      // The next step's units have come (what may still be on its way: those behind that), and nobody reads this step's any more.
      if (i == kHold) {
        wait(std::integral_constant<int, O::loads * (2 * S::ahead - 3)>{});
      }
      constexpr int kLeft = S::FI - kHold;
      const int at = i - kHold;
#pragma unroll
      for (int k = at * kSoon; k < std::min((at + 1) * kSoon, S::FJ); ++k) read_b(k, 0, next_b);
      if (i == kHold) {
#pragma unroll
        for (int k = 0; k < kHold; ++k) read_a(k, 0, next_a);
      }
      read_a(i, 0, next_a);
#pragma unroll
      for (int k = at * O::loads / kLeft; k < (at + 1) * O::loads / kLeft; ++k) ob.load(k, start + ua, ahead, last);
      __builtin_amdgcn_sched_barrier(0);
    }
    ua = next_a;
  }

  // The tile's end, one strip of blocks after the other, by code that is there once (a workgroup runs it once, at the pace at which
  // instructions come from memory: unrolled it took 10 us more).  Scales and bias go through LDS, behind the strips; the residual's
  // values are asked for four turns ahead.
  constexpr int N = std::is_same_v<T, float> ? 4 : 8;
  using P = Strips<S::FI / 2, S::FJ / 2, S::WI, S::WJ, N>;
  constexpr int kStrips = S::WI * S::WJ * P::bytes;
  static_assert(kStrips + 3 * S::B * 4 <= S::units * S::unit && S::threads >= S::B, "the strips have to fit the operands' place");
  typedef __attribute__((address_space(3))) float lds_float;
  lds_char* const strip = all + wave * P::bytes;
  lds_float* const scales = (lds_float*)(all + kStrips);
  auto ready = [&]() {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };
  auto sum_of = [&](int (&sum)[N], int turn) {
    float v[N];
    P::get(v, strip, turn, lane);
    __builtin_memcpy(sum, v, sizeof v);
  };
  auto put = [&](int q) {
#pragma unroll
    for (int k = 0; k < S::FJ; ++k) {
      if (k / 2 != q) continue;
#pragma unroll
      for (int i = 0; i < S::FI; ++i) *reinterpret_cast<lds_i32x4*>(strip + P::place(k % 2 * 16 + (lane & 15), 4 * i + (lane >> 4))) = acc[i][k];
    }
  };
  auto end = [&](auto&& others) {
    ready();
    if (t < S::B) scales[t] = of_a, scales[S::B + t] = of_b, scales[2 * S::B + t] = of_bias;
    ready();
    const int i = P::column(wave * P::per_wave, lane), n = a.ni - i0 - i;
    float scale[N], bias[N];
#pragma unroll
    for (int k = 0; k < N; ++k) scale[k] = scales[i + k], bias[k] = scales[2 * S::B + i + k];
    constexpr int kAhead = 4;
    // rows follow each other from turn to turn and from strip to strip
    const int row = P::row(wave * P::per_wave, lane), left = n > 0 ? (int)min(a.nj - j0, (int64_t)S::B) - row : 0;      // rows from here on
    T* out = static_cast<T*>(a.out) + (j0 + row) * a.ldo + i0 + i;
    const T* from = static_cast<const T*>(a.residual) + (j0 + row) * a.ldr + i0 + i;
    float residual[kAhead][N] = {};
    auto ask = [&](float (&r)[N], int turn) {
      if (!a.residual) return;
      load_values(r, from, turn * P::rows < left ? n : 0);
      from += P::rows * a.ldr;
    };
#pragma unroll
    for (int k = 0; k < kAhead - 1; ++k) ask(residual[k], k);
#pragma clang loop unroll(disable)
    for (int q = 0; q < S::FJ / 2; ++q) {
      put(q);
#pragma clang loop unroll(disable)
      for (int turn = 0; turn < P::turns; ++turn) {
        const int at = q * P::turns + turn;
        ask(residual[kAhead - 1], at + kAhead - 1);
        int sum[N];
        sum_of(sum, turn);
        others(sum, wave * P::per_wave + at);
        const float by = scales[S::B + row + at * P::rows];
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = fmaf((float)sum[k], by * scale[k], bias[k]);
        activate_all(v, a.act);
        if (a.residual) {
#pragma unroll
          for (int k = 0; k < N; ++k) v[k] += residual[0][k];
#pragma unroll
          for (int c = 0; c + 1 < kAhead; ++c)
#pragma unroll
            for (int k = 0; k < N; ++k) residual[c][k] = residual[c + 1][k];
        }
        if (at * P::rows < left) store_values(out, v, n);
        out += P::rows * a.ldo;
      }
    }
  };
  if (sp.splits == 1) {
    end([](int (&)[N], int) {});
    return;
  }
  // A sum in parts: each workgroup leaves its part, lanes side by side, and the one that comes last to a tile adds the others' to its own
  // (integers: in any order).  Parts are stored and read with agent-scope atomics, which go past the caches that the XCDs do not share:
  // every store has arrived when vmcnt says so, and the barrier puts all of the workgroup's before its count.
  const int tile = at.tj * sp.tiles_i + at.ti, tiles = sp.tiles_i * sp.tiles_j;
  auto part = [&](int split, int piece) {
    return static_cast<uint64_t*>(a.workspace) + (((int64_t)split * tiles + tile) * P::pieces + piece) * (64 * N / 2) + lane;
  };
  ready();
#pragma clang loop unroll(disable)
  for (int q = 0; q < S::FJ / 2; ++q) {
    put(q);
#pragma clang loop unroll(disable)
    for (int turn = 0; turn < P::turns; ++turn) {
      int sum[N];
      sum_of(sum, turn);
      uint64_t x[N / 2], *to = part(at.split, wave * P::per_wave + q * P::turns + turn);
      __builtin_memcpy(x, sum, sizeof sum);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) __hip_atomic_store(to + 64 * k, x[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
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
  end([&](int (&sum)[N], int piece) {
    for (int k = 0; k < sp.splits; ++k) {
      if (k == at.split) continue;
      const uint64_t* from = part(k, piece);
      uint64_t x[N / 2];
      int other[N];
#pragma unroll
      for (int c = 0; c < N / 2; ++c) x[c] = __hip_atomic_load(from + 64 * c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __builtin_memcpy(other, x, sizeof other);
#pragma unroll
      for (int c = 0; c < N; ++c) sum[c] += other[c];
    }
  });
}

// The same for few samples: a workgroup has 16 FI x 16 FJ of D, its wavefronts a run of the depth each, whose operands come from memory as
// v_mfma_i32_16x16x64_i8 takes them, U steps of 64 on their way.  The sums meet in LDS.  Bound by how soon the weight's rows are there, not by its stream:
// 16 x 4096 -> 4096 6.9 us (2.4 TB/s), 2.6 of which do not depend on the size.
template <typename T, int FI, int FJ, int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void int8_few_kernel(Int8Args a, int tiles_i, int tiles_j) {
  // workgroups go round the 8 XCDs: tiles of the same weight rows follow each other on one where there are rows for all, as the grid has it
  const bool rows_first = tiles_i >= 64;
  const int q = (int)blockIdx.x >> 3, ti = rows_first ? q / tiles_j * 8 + ((int)blockIdx.x & 7) : (int)blockIdx.x % tiles_i;
  const int tj = rows_first ? q % tiles_j : (int)blockIdx.x / tiles_i;
  if (ti >= tiles_i || tj >= tiles_j) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = ti * 16 * FI;
  const int64_t j0 = (int64_t)tj * 16 * FJ;
  const int at = 16 * (lane >> 4), steps = (a.stride + 63) / 64, each = (steps + WAVES - 1) / WAVES;
  const int first = min(wave * each, steps) * 64, end = min((wave + 1) * each, steps) * 64;
  const int8_t* pa[FI];
  const int8_t* pb[FJ];
#pragma unroll
  for (int k = 0; k < FI; ++k) pa[k] = a.a + (int64_t)min(i0 + 16 * k + (lane & 15), a.ni - 1) * a.stride;
#pragma unroll
  for (int k = 0; k < FJ; ++k) pb[k] = a.b + min(j0 + 16 * k + (lane & 15), a.nj - 1) * a.stride;
  // a wavefront ends a block: asked for before the sums
  static_assert(FI * FJ <= WAVES);
  const int64_t j = j0 + wave % FJ * 16 + (lane & 15);
  const int i = i0 + wave / FJ * 16 + 4 * (lane >> 4);
  End<T, 4> e;
  if (wave < FI * FJ) e.load(a, j, i);
  i32x4 acc[FI][FJ] = {};
  for (int r = first; r < end; r += 64 * U) {
    i32x4 va[U][FI], vb[U][FJ];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // beyond the end of the run or of the row: read again what is there, and not used
      const int col = min(r + 64 * u, end - 64) + at, in = min(col, a.stride - 16);
#pragma unroll
      for (int k = 0; k < FI; ++k) va[u][k] = *reinterpret_cast<const i32x4*>(pa[k] + in);
#pragma unroll
      for (int k = 0; k < FJ; ++k) vb[u][k] = *reinterpret_cast<const i32x4*>(pb[k] + in);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = r + 64 * u < end && r + 64 * u + at < a.stride;
#pragma unroll
      for (int k = 0; k < FI; ++k) {
        const i32x4 v = there ? va[u][k] : i32x4{};
#pragma unroll
        for (int c = 0; c < FJ; ++c) acc[k][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, vb[u][c], acc[k][c], 0, 0, 0);
      }
    }
  }
  __shared__ i32x4 sums[WAVES][FI * FJ][64];
#pragma unroll
  for (int k = 0; k < FI; ++k)
#pragma unroll
    for (int c = 0; c < FJ; ++c) sums[wave][k * FJ + c][lane] = acc[k][c];
  __syncthreads();
  if (wave >= FI * FJ) return;
  i32x4 total = sums[0][wave][lane];
#pragma unroll
  for (int k = 1; k < WAVES; ++k) total += sums[k][wave][lane];
  const int sum[4] = {total[0], total[1], total[2], total[3]};
  e.finish(sum, a, j, i);
}

// A single token: the four wavefronts of a workgroup share two weight rows, which they read in runs of 1024 codes, 16 a lane, in turn, U runs on
// their way, and multiply by v_dot4.  The lanes' sums are added up at the end, the wavefronts' in LDS.  Bound by the weight's stream: 4096 ->
// 11008 9.2 us (4.9 TB/s with the launch), 8192 -> 8192 12.4 (5.4).  Tried: one, three, four, six and eight rows, and rows to a wavefront or two
// (4096 -> 11008 9.5 to 16.5 us).
template <typename T, int U>
__global__ __launch_bounds__(256) void int8_token_kernel(Int8Args a) {
  constexpr int R = 2, D = 4;
  const int lane = threadIdx.x & 63, slice = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = (int)blockIdx.x * R, i = lane < R ? i0 + lane : a.ni;
  End<T, 1> e;
  if (slice == 0) e.load(a, 0, i);
  const int8_t* row[R];
#pragma unroll
  for (int k = 0; k < R; ++k) row[k] = a.a + (int64_t)min(i0 + k, a.ni - 1) * a.stride;
  int acc[R] = {};
  for (int r = 1024 * slice; r < a.stride; r += 1024 * U * D) {
    i32x4 w[U][R], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int in = min(r + 1024 * u * D + 16 * lane, a.stride - 16);
#pragma unroll
      for (int k = 0; k < R; ++k) w[u][k] = *reinterpret_cast<const i32x4*>(row[k] + in);
      x[u] = *reinterpret_cast<const i32x4*>(a.b + in);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const i32x4 v = r + 1024 * u * D + 16 * lane < a.stride ? x[u] : i32x4{};
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[k] = __builtin_amdgcn_sdot4(w[u][k][c], v[c], acc[k], false);
    }
  }
  int sum[1] = {0};
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int total = over_wave(acc[k], Plus{});
    if (lane == k) sum[0] = total;
  }
  __shared__ int sums[D][R];
  if (lane < R) sums[slice][lane] = sum[0];
  __syncthreads();
  if (slice > 0 || lane >= R) return;
#pragma unroll
  for (int k = 1; k < D; ++k) sum[0] += sums[k][lane];
  e.finish(sum, a, 0, i);
}

template <typename T, typename S>
hipError_t run_product(const Int8Args& a, const Split& sp, hipStream_t s) {
  int8_product_kernel<T, S><<<dim3((unsigned)((int64_t)sp.tiles_i * sp.tiles_j * sp.splits)), S::threads, 0, s>>>(a, sp);
  return hipGetLastError();
}
template <typename T, int FJ>
hipError_t run_few(const Int8Args& a, const Split& sp, hipStream_t s) {
  int8_few_kernel<T, 1, FJ, 8, 2><<<dim3((unsigned)((sp.tiles_i + 7) / 8 * 8 * sp.tiles_j)), 512, 0, s>>>(a, sp.tiles_i, sp.tiles_j);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_product(int type, const Int8Args& a, hipStream_t s) {
  const Int8Plan p = plan_int8(a.ni, a.nj, a.stride);
  if (p.us < 0.f) return hipErrorInvalidValue;
  return by_type(type, [&](auto zero) {
    using T = decltype(zero);
    switch (p.kernel) {
      case kToken:
        // a run a wavefront where there is no second (us, one run / two on their way: 4096 -> 11008 9.2 / 9.7, 11008 -> 4096 11.4 / 10.1)
        if (a.stride <= 4096) int8_token_kernel<T, 1><<<dim3((unsigned)p.sp.tiles_i), 256, 0, s>>>(a);
        else int8_token_kernel<T, 2><<<dim3((unsigned)p.sp.tiles_i), 256, 0, s>>>(a);
        return hipGetLastError();
      case kFew16: return run_few<T, 1>(a, p.sp, s);
      case kFew32: return run_few<T, 2>(a, p.sp, s);
      case kTile64: return p.deep ? run_product<T, Shape<64, 2, 2, 4>>(a, p.sp, s) : run_product<T, Shape<64, 2, 2, 2>>(a, p.sp, s);
      case kTile128: return p.deep ? run_product<T, Shape<128, 2, 4, 4>>(a, p.sp, s) : run_product<T, Shape<128, 2, 4, 2>>(a, p.sp, s);
      default: return run_product<T, Shape<256, 2, 4, 2>>(a, p.sp, s);
    }
  });
}

}  // namespace linear
}  // namespace lqsgd
