// Which kernel a product of 8-bit rows takes, and in how many parts its sum.  Host only, no HIP.
#pragma once

#include <algorithm>
#include <cstdint>

#include "lqsgd_linear_plan.h"

namespace lqsgd {
namespace linear {

enum Int8Kernel { kToken = 0, kFew16, kFew32, kTile64, kTile128, kTile256, kInt8Kernels };
constexpr int kDeep = 128;                  // codes of a step of the tiles' kernels

struct Int8Plan {
  Int8Kernel kernel;
  Split sp;
  bool deep;             // kTile64, kTile128: four steps of operands in LDS, not two
  float us;              // expected
};

// D is nj x ni, rows of `stride` codes.  One sample has a kernel of its own; otherwise the kernel with the least expected time of
//   few samples (a workgroup reads 16 rows of the weight and 16 or 32 samples whole)   2.6 us + 2.2 us a 1000 workgroups + the larger of
//     all that at 8 TB/s and 0.3 us + 0.5 us a 1000 codes (32 samples: 0.8 and 0.75)
//   64 x 64     4.4 us + steps 0.235 us with one workgroup a CU, 4.4 us + 0.6 us a further turn + turns steps 0.19 us with more
//   128 x 128   5.5 us + steps (0.33 + 0.2 w), 5.5 us + 2.5 us a further turn + turns steps 0.46 us
//   256 x 256   1.5 us + turns (10 us + steps (0.93 + 0.57 w))
// for turns of 256 workgroups, w = the share of the 256 CUs that have a workgroup, and for a sum in parts 1.5 us + 1.1 us a part + 0.25 us a MiB of them.  Fits to
// the kernels' times over 45 products from 1 x 512 x 512 to 8192 x 4096 x 4096 in bfloat16; over 63 others its choices are 1 to 3 % above the best kernels'
// times on average, 36 % at worst (1735 x 6526 -> 18 12.2 us, not 9.0).  E.g. (us, samples x cols -> rows: few / 64 / 128 / 256)
// 16 x 4096 -> 4096 6.9 / 11.7 / - / -, 64 x 4096 -> 11008 36.8 / 14.1 / 30 / -, 256 x 4096 -> 4096 - / 12.7 / 17.0 / 42,
// 1024 x 4096 -> 4096 - / 28.5 / 20.6 / 42, 4096 x 11008 -> 4096 - / 297 / 186 / 146; 64 x 11008 -> 4096 in four parts 16.6, whole 28.6.
// Operands of four steps in LDS leave room for half as many workgroups on a CU: for as many as there is room for, and sums of eight steps or
// more (1024 x 4096 -> 4096 20.6 / 22.9 with two steps, 2048 x 4096 -> 4096 40.4 / 36.9; 1402 x 175 -> 701 by 64 x 64 5.7 / 5.2).
inline Int8Plan plan_int8(int64_t ni, int64_t nj, int64_t stride) {
  Int8Plan best{};
  best.us = -1.f;
  auto offer = [&](Int8Kernel k, int64_t ti, int64_t tj, int splits, int64_t per, bool deep, float us) {
    if (best.us >= 0.f && us >= best.us) return;
    best = Int8Plan{k, Split{(int)ti, (int)tj, splits, per * kDeep}, deep, us};
  };
  const int64_t steps = (stride + kDeep - 1) / kDeep;
  if (nj <= 1) {
    offer(kToken, (ni + 1) / 2, 1, 1, steps, false, 0.f);
    return best;
  }
  for (int f = 0; f < 2; ++f) {
    const int64_t bj = f ? 32 : 16, ti = (ni + 15) / 16, tj = (nj + bj - 1) / bj;
    if ((ti + 7) / 8 * 8 * tj >= 1 << 20) continue;                        // as many workgroups, of 512 threads
    const float all = (float)(ti * tj) * (float)((16 + bj) * stride) / 8e6f, one = (f ? .8f : .3f) + (float)stride * (f ? .75e-3f : .5e-3f);
    offer(f ? kFew32 : kFew16, ti, tj, 1, steps, false, 2.6f + 2.2e-3f * (float)(ti * tj) + std::max(all, one));
  }
  for (int k = 0; k < 3; ++k) {
    const int64_t b = 64 << k, ti = (ni + b - 1) / b, tj = (nj + b - 1) / b, tiles = ti * tj;
    if (tiles * (k ? 512 : 256) >= int64_t(1) << 32) continue;            // a launch has fewer threads
    for (int parts = 1; parts <= 8; ++parts) {
      if (parts > 1 && (parts > steps || tiles > kTiles || tiles * parts * b * b * 4 > (int64_t)kWorkspaceBytes)) break;
      const int64_t per = (steps + parts - 1) / parts, groups = tiles * parts, turns = (groups + 255) / 256;
      if (parts > 1 && (steps + per - 1) / per != parts) continue;        // as many steps a part as with fewer parts
      const float w = std::min(1.f, (float)groups / 256.f), n = (float)per;
      const float t = (float)turns;
      float us = k == 0 ? (turns > 1 ? 4.4f + .6f * (t - 1.f) + .19f * t * n : 4.4f + .235f * n)
               : k == 1 ? (turns > 1 ? 5.5f + 2.5f * (t - 1.f) + .46f * t * n : 5.5f + (.33f + .2f * w) * n)
                        : 1.5f + t * (10.f + n * (.93f + .57f * w));
      if (parts > 1) us += 1.5f + 1.1f * (float)parts + .25f * (float)(groups * b * b * 4) / 1048576.f;
      offer(k == 0 ? kTile64 : k == 1 ? kTile128 : kTile256, ti, tj, parts, per, per >= 8 && groups <= (k == 0 ? 512 : 256), us);
    }
  }
  return best;
}

}  // namespace linear
}  // namespace lqsgd
