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


# Products that reach each kernel, with the sum whole and in parts, several steps deep and with remainders in every direction: (product,
# operands, samples, rows, cols, kernel, in parts).  operands: "f32"; "direct", 16 bits straight into LDS; "any", 16 bits of any length.
CASES = [
    ("forward", "f32", 201, 8199, 203, "128 x 128", False), ("forward", "f32", 8201, 73, 521, "128 x 128", True),
    ("forward", "f32", 1545, 2570, 201, "large", False), ("forward", "f32", 201, 8201, 523, "large", True),
    ("forward", "f32", 41, 43, 201, "by depth", False), ("forward", "f32", 41, 39, 1305, "by depth", True),
    ("forward", "f32", 3, 1001, 130, "by depth", False), ("forward", "f32", 3, 1001, 2049, "by depth", True),
    ("forward", "direct", 73, 8201, 200, "128 x 128", False), ("forward", "direct", 41, 39, 2568, "128 x 128", True),
    ("forward", "direct", 1305, 6151, 328, "large", False), ("forward", "direct", 201, 8201, 4104, "large", True),
    ("forward", "direct", 41, 39, 200, "by depth", False), ("forward", "direct", 39, 41, 8200, "by depth", True),
    ("forward", "direct", 3, 1001, 520, "by depth", False), ("forward", "direct", 1, 1001, 8200, "by depth", True),
    ("forward", "any", 73, 8201, 201, "128 x 128", False), ("forward", "any", 73, 8201, 521, "128 x 128", True),
    ("forward", "any", 1545, 2569, 201, "large", False), ("forward", "any", 73, 8201, 1305, "large", True),
    ("forward", "any", 41, 39, 201, "by depth", False), ("forward", "any", 39, 41, 1545, "by depth", True),
    ("forward", "any", 3, 1001, 513, "by depth", False), ("forward", "any", 1, 1001, 4099, "by depth", True),
    ("input_grad", "f32", 201, 203, 8199, "128 x 128", False), ("input_grad", "f32", 8201, 521, 73, "128 x 128", True),
    ("input_grad", "f32", 1545, 201, 2570, "large", False), ("input_grad", "f32", 201, 523, 8201, "large", True),
    ("input_grad", "f32", 41, 201, 43, "by depth", False), ("input_grad", "f32", 41, 1305, 39, "by depth", True),
    ("input_grad", "f32", 3, 130, 1001, "by depth", False), ("input_grad", "f32", 3, 2049, 1001, "by depth", True),
    ("input_grad", "direct", 73, 200, 8200, "128 x 128", False), ("input_grad", "direct", 41, 2568, 40, "128 x 128", True),
    ("input_grad", "direct", 1305, 328, 6152, "large", False), ("input_grad", "direct", 201, 4104, 8200, "large", True),
    ("input_grad", "direct", 41, 200, 40, "by depth", False), ("input_grad", "direct", 39, 8200, 40, "by depth", True),
    ("input_grad", "direct", 3, 520, 1000, "by depth", False), ("input_grad", "direct", 1, 8200, 1000, "by depth", True),
    ("input_grad", "any", 73, 201, 8201, "128 x 128", False), ("input_grad", "any", 73, 521, 8201, "128 x 128", True),
    ("input_grad", "any", 1545, 201, 2569, "large", False), ("input_grad", "any", 73, 1305, 8201, "large", True),
    ("input_grad", "any", 41, 201, 39, "by depth", False), ("input_grad", "any", 39, 1545, 41, "by depth", True),
    ("input_grad", "any", 3, 513, 1001, "by depth", False), ("input_grad", "any", 1, 4099, 1001, "by depth", True),
    ("weight_grad", "f32", 203, 201, 8199, "128 x 128", False), ("weight_grad", "f32", 1033, 8201, 73, "128 x 128", True),
    ("weight_grad", "f32", 201, 1545, 2570, "large", False), ("weight_grad", "f32", 523, 201, 8201, "large", True),
    ("weight_grad", "f32", 201, 43, 39, "by depth", False), ("weight_grad", "f32", 1033, 41, 39, "by depth", True),
    ("weight_grad", "f32", 130, 3, 1001, "by depth", False), ("weight_grad", "f32", 2049, 3, 1001, "by depth", True),
    ("weight_grad", "direct", 201, 72, 8201, "128 x 128", False), ("weight_grad", "direct", 1033, 72, 8201, "128 x 128", True),
    ("weight_grad", "direct", 327, 1544, 2570, "large", False), ("weight_grad", "direct", 1545, 200, 8201, "large", True),
    ("weight_grad", "direct", 201, 40, 39, "by depth", False), ("weight_grad", "direct", 2057, 40, 41, "by depth", True),
    ("weight_grad", "direct", 513, 8, 1001, "by depth", False), ("weight_grad", "direct", 4099, 8, 1001, "by depth", True),
    ("weight_grad", "any", 201, 73, 8201, "128 x 128", False), ("weight_grad", "any", 521, 73, 8201, "128 x 128", True),
    ("weight_grad", "any", 201, 1545, 2569, "large", False), ("weight_grad", "any", 1305, 73, 8201, "large", True),
    ("weight_grad", "any", 201, 41, 39, "by depth", False), ("weight_grad", "any", 1545, 41, 39, "by depth", True),
    ("weight_grad", "any", 513, 3, 1001, "by depth", False), ("weight_grad", "any", 4099, 3, 1001, "by depth", True),
]
