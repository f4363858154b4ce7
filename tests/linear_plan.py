"""csrc/lqsgd_linear_plan.h from Python: which kernel the library takes for a product of the linear layer.  A few lines of C++ around the
header, built with the host compiler; no GPU."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PRODUCTS = ("forward", "input_grad", "weight_grad")
KERNELS = ("by depth", "128 x 128", "large")
PROGRAM = r"""
#include <cinttypes>
#include <cstdio>
#include "lqsgd_linear_plan.h"
int main() {
  int product, fp32, direct;
  int64_t ni, nj, depth;
  while (std::scanf("%d %d %d %" SCNd64 " %" SCNd64 " %" SCNd64, &product, &fp32, &direct, &ni, &nj, &depth) == 6) {
    const lqsgd::linear::Plan p = lqsgd::linear::plan_product(product, fp32 != 0, direct != 0, ni, nj, depth);
    std::printf("%d %d %d %d %" PRId64 " %" PRId64 "\n", (int)p.kernel, p.sp.splits, p.sp.tiles_i, p.sp.tiles_j, p.sp.steps, p.tiles);
  }
}
"""


def compiler():
    return shutil.which("g++") or shutil.which("c++")


def build(folder):
    src, exe = os.path.join(str(folder), "plan.cpp"), os.path.join(str(folder), "plan")
    with open(src, "w") as fh:
        fh.write(PROGRAM)
    subprocess.run([compiler(), "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2506_17974_amd", "csrc"),
                    src, "-o", exe], check=True)
    return exe


def is_direct(product, kind, samples, rows, cols):
    """Whether dense 16-bit operands go straight into LDS: all of their rows are whole chunks of 8."""
    runs = {"forward": (cols,), "input_grad": (cols, rows), "weight_grad": (rows,)}[product]
    return kind != "f32" and all(r % 8 == 0 for r in runs)


def plans(exe, asked):
    """[(kernel, parts, tiles_i, tiles_j, steps, tiles)] for [(product, kind, samples, rows, cols)] of dense, aligned tensors."""
    lines = []
    for product, kind, m, n, k in asked:
        ni, nj, depth = {"forward": (n, m, k), "input_grad": (k, m, n), "weight_grad": (k, n, m)}[product]
        lines.append("%d %d %d %d %d %d" % (PRODUCTS.index(product), kind == "f32", is_direct(product, kind, m, n, k), ni, nj, depth))
    out = subprocess.run([exe], input="\n".join(lines) + "\n", stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
    got = [tuple(int(v) for v in line.split()) for line in out if line]
    assert len(got) == len(asked)
    return [(KERNELS[g[0]],) + g[1:] for g in got]
