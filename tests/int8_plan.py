"""csrc/lqsgd_int8_plan.h from Python: which kernel the library takes for a product of 8-bit rows.  A few lines of C++ around the header,
built with the host compiler; no GPU."""
import os
import subprocess

from tests.linear_plan import ROOT, compiler

KERNELS = ("token", "few 16", "few 32", "64", "128", "256")
PROGRAM = r"""
#include <cinttypes>
#include <cstdio>
#include "lqsgd_int8_plan.h"
int main() {
  int64_t samples, rows, cols;
  while (std::scanf("%" SCNd64 " %" SCNd64 " %" SCNd64, &samples, &rows, &cols) == 3) {
    const lqsgd::linear::Int8Plan p = lqsgd::linear::plan_int8(rows, samples, (cols + 31) / 32 * 32);
    std::printf("%d %d %d %d %d %" PRId64 " %g\n", (int)p.kernel, (int)p.deep, p.sp.splits, p.sp.tiles_i, p.sp.tiles_j, p.sp.steps, p.us);
  }
}
"""


def build(folder):
    src, exe = os.path.join(str(folder), "plan.cpp"), os.path.join(str(folder), "plan")
    with open(src, "w") as fh:
        fh.write(PROGRAM)
    subprocess.run([compiler(), "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2506_17974_amd", "csrc"),
                    src, "-o", exe], check=True)
    return exe


def plans(exe, asked):
    """[(kernel, deep, parts, tiles_i, tiles_j, codes of a part, us)] for [(samples, rows, cols)]."""
    out = subprocess.run([exe], input="\n".join("%d %d %d" % a for a in asked) + "\n", stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
    got = [line.split() for line in out if line]
    assert len(got) == len(asked)
    return [(KERNELS[int(g[0])], g[1] == "1") + tuple(int(v) for v in g[2:6]) + (float(g[6]),) for g in got]


# Products that reach each kernel, with operands of two and of four steps in LDS, the sum whole and in parts, remainders in every
# direction: (samples, rows, cols, kernel, four steps, in parts).  "few" kernels go by the weight's rows first from 64 tiles of them on.
CASES = [
    (1, 1, 1, "token", False, False), (1, 4099, 2051, "token", False, False), (1, 5, 9001, "token", False, False),
    (3, 37, 1001, "few 16", False, False), (15, 1049, 67, "few 16", False, False), (3, 1049, 4099, "few 16", False, False),
    (2991, 39, 1193, "few 32", False, False), (107, 826, 1576, "few 32", False, False), (29, 4459, 335, "few 32", False, False),
    (35, 4946, 370, "64", False, False), (4, 8645, 2299, "64", True, False), (3, 7144, 7475, "64", True, True),
    (1198, 1705, 263, "128", False, False), (452, 4140, 1026, "128", True, False), (101, 8407, 5074, "128", True, True), (7670, 581, 8903, "128", False, True),
    (6532, 1864, 265, "256", False, False), (2115, 1999, 6843, "256", True, True),
]
