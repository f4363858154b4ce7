// Which kernel a product of the linear layer takes, and how its sum is shared out.  Host only, no HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace lqsgd {
namespace linear {

// A product D[j][i] = sum over r < depth of A[i][r] B[j][r], i < ni contiguous in the output's rows, j < nj its rows:
//   forward       i = output feature  A = w    (r contiguous)   j = sample          B = x  (r contiguous)   r = input feature
//   input grad    i = input feature   A = w    (i contiguous)   j = sample          B = dz (r contiguous)   r = output feature
//   weight grad   i = input feature   A = x^   (i contiguous)   j = output feature  B = dz (j contiguous)   r = sample
enum Product { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

constexpr size_t kWorkspaceBytes = 64ull << 20;   // sums of parts, at most
constexpr int kTiles = 8192;                      // tiles whose sum is in parts, at most (64 x 32, two parts)

// A tile's sum in `splits` parts.
struct Split {
  int tiles_i, tiles_j, splits;
  int64_t steps;         // values of r of a split, a multiple of the kernel's step
};

// Three kernels serve a product: by depth (64 x 64 tiles, the sum shared out among a workgroup's wavefronts), 128 x 128 tiles and
// the largest ones, each with the sum whole or in parts that are added up at the end.  The one with the least expected time is taken:
//   1.5 us + turns (turn + steps (step + more w)) + [parts > 1] (4 us + what the join writes and reads at 4.5 TB/s)
// for `turns` rounds of 256 workgroups of `steps` steps each and w = the share of the CUs that have one; by depth, where one workgroup
// adds up a tile, 0.35 us a part more.  The figures are fits to the three kernels' times over 120 products from 64 x 1024 x 64 to
// 8192 x 2048 x 1024 in bfloat16 and fp32; taken by them the products cost 2 % more than each one's best.  E.g. (bf16,
// ni x nj x depth: by depth / 128 x 128 / 256 x 256) 1024 x 1024 x 1024 8 / 16 / 29 us, 2048 x 2048 x 2048 39 / 28 / 50,
// 4096 x 4096 x 512 72 / 28 / 23; fp32 512 x 4096 x 4096 139 / 240 / 283, in 4 parts by the last 100.
struct Rate { float turn, step, more; };
enum Kernel { kByDepth = 0, kMiddle = 1, kLarge = 2 };
struct Plan {
  Kernel kernel;
  Split sp;
  int64_t tiles;         // 0: no kernel can be launched with so many
};
struct Geometry { int bi, bj, step, threads; };

// fp32: operands of 32 bits; direct: 16-bit operands of whole aligned chunks, which go straight into LDS.
inline Plan plan_product(int product, bool fp32, bool direct, int64_t ni, int64_t nj, int64_t depth) {
  const bool grad = product == kWeightGrad;
  const Rate rates[3] = {fp32 ? grad ? Rate{2.8f, 1.15f, .2f} : Rate{3.2f, 1.65f, .35f}
                              : direct ? grad ? Rate{3.6f, 1.5f, .35f} : Rate{3.4f, 1.f, .45f} : Rate{3.6f, 2.2f, .6f},
                         fp32 ? grad ? Rate{6.f, 1.35f, .05f} : Rate{8.f, 1.85f, .05f}
                              : direct ? grad ? Rate{4.f, .58f, .12f} : Rate{2.8f, .34f, 0.f} : Rate{5.f, .9f, .1f},
                         fp32 ? grad ? Rate{6.5f, 1.36f, .1f} : Rate{8.f, 2.f, .5f}
                              : direct ? grad ? Rate{9.f, .78f, .22f} : Rate{9.f, .62f, .25f} : Rate{8.f, .8f, .1f}};
  const Geometry shapes[3] = {{64, nj <= 32 ? 32 : 64, fp32 ? nj <= 32 ? 256 : 128 : 512, 512},
                              {128, 128, 32, 256},
                              {256, !fp32 && direct ? 256 : 128, 32, 512}};
  Plan best{};
  float least = 0.f;
  for (int k = 0; k < 3; ++k) {
    const Geometry& g = shapes[k];
    const int64_t ti = (ni + g.bi - 1) / g.bi, tj = (nj + g.bj - 1) / g.bj, tiles = ti * tj, steps = (depth + g.step - 1) / g.step;
    if (tiles * g.threads >= int64_t(1) << 32) continue;                   // a launch has fewer threads
    const int64_t fit = (int64_t)(kWorkspaceBytes / (sizeof(float) * g.bi * g.bj)) / tiles;
    for (int64_t parts = 1; parts <= 16; ++parts) {
      if (parts > 1 && (parts > steps || parts > fit)) break;
      const int64_t per = parts > 1 ? (steps + parts - 1) / parts : steps;
      if (parts > 1 && (steps + per - 1) / per != parts) continue;         // as many steps a part as with fewer parts
      const int64_t groups = tiles * parts, turns = (groups + 255) / 256;
      const Rate& r = rates[k];
      float us = 1.5f + (float)turns * (r.turn + (float)per * (r.step + r.more * std::min(1.f, (float)groups / 256.f)));
      if (parts > 1) us += 4.f + 4e-6f / 4.5f * (float)(groups * g.bi * g.bj) + (k == kByDepth ? .35f * (float)parts : 0.f);
      if (best.tiles == 0 || us < least) {
        least = us;
        best.kernel = (Kernel)k;
        best.sp = Split{(int)ti, (int)tj, (int)parts, std::max<int64_t>(1, per) * g.step};
        best.tiles = tiles;
      }
    }
  }
  return best;
}

}  // namespace linear
}  // namespace lqsgd
