"""CPU-only checks of the rule that gives each product of the linear layer its kernel."""
import pytest

from tests import linear_plan as lp

pytestmark = pytest.mark.skipif(lp.compiler() is None, reason="no C++ compiler")
THREADS = {"by depth": 512, "128 x 128": 256, "large": 512}
TILE = {"by depth": (64, 64), "128 x 128": (128, 128)}


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return lp.build(tmp_path_factory.mktemp("plan"))


def _check(asked, p):
    """A plan that covers its output and depth and that one launch holds."""
    product, kind, m, n, k = asked
    kernel, parts, ti, tj, steps, tiles = p
    ni, nj, depth = {"forward": (n, m, k), "input_grad": (k, m, n), "weight_grad": (k, n, m)}[product]
    bi, bj = TILE.get(kernel, (256, 256 if lp.is_direct(*asked) else 128))
    if kernel == "by depth" and nj <= 32:
        bj = 32
    assert tiles == ti * tj > 0, asked
    assert (ti - 1) * bi < ni <= ti * bi and (tj - 1) * bj < nj <= tj * bj, (asked, p)
    assert tiles * parts * THREADS[kernel] < 1 << 32, (asked, p)
    assert (parts - 1) * steps < max(depth, 1) <= parts * steps and steps % 16 == 0, (asked, p)
    assert parts == 1 or tiles * parts * bi * bj * 4 <= 64 << 20 and tiles <= 8192, (asked, p)


def test_every_size_in_range_has_a_kernel(exe):
    """Up to 2^30 samples, 2^20 features and 2^36 values of the output."""
    top = 1 << 30
    asked = []
    for kind in ("f32", "bf16"):
        for m in (1, 31, 33, 1000, 1 << 16, (1 << 22) + 5, (1 << 27) - 1, 1 << 28, 1 << 29, top - 1, top):
            for n in (1, 8, 16, 32, 63, 64, 65, 127, 128, 129, 256, 1000, 1 << 14, 1 << 20):
                for k in (1, 16, 64, 129, 4096, 1 << 20):
                    if m * n <= 1 << 36:
                        asked.append(("forward", kind, m, n, k))
                        asked.append(("input_grad", kind, m, k, n))
                    if n * k <= 1 << 36:
                        asked.append(("weight_grad", kind, m, n, k))
    for a, p in zip(asked, lp.plans(exe, asked)):
        _check(a, p)


def test_what_no_launch_holds_is_said(exe):
    """The limits differ with the tiles: beyond all of them there is no plan, and none is made up."""
    top = 1 << 30
    assert [p[5] for p in lp.plans(exe, [("forward", "f32", top, 1 << 20, 1), ("input_grad", "bf16", top, 1, 1 << 20)])] == [0, 0]
    narrow = lp.plans(exe, [("forward", "bf16", top, 16, 16), ("forward", "f32", top, 64, 64)])
    assert [p[0] for p in narrow] == ["128 x 128"] * 2 and [p[5] for p in narrow] == [1 << 23] * 2


def test_the_gpu_tests_reach_every_kernel(exe):
    """The products of lp.CASES are served by the kernels that they are listed for, and every one of those is there."""
    asked = [(product, "f32" if operands == "f32" else "bf16", m, n, k) for product, operands, m, n, k, _, _ in lp.CASES]
    covered = set()
    for case, a, p in zip(lp.CASES, asked, lp.plans(exe, asked)):
        product, operands, m, n, k, kernel, in_parts = case
        assert operands == ("f32" if a[1] == "f32" else "direct" if lp.is_direct(*a) else "any"), case
        assert (p[0], p[1] > 1) == (kernel, in_parts), (case, p)
        _check(a, p)
        nj = {"forward": m, "input_grad": m, "weight_grad": n}[product]
        depth = {"forward": k, "input_grad": n, "weight_grad": m}[product]
        if kernel != "by depth":
            assert min(p[4], depth) > 5 * 32, (case, p)         # more steps than there are buffers
        covered.add((product, operands, kernel, in_parts, kernel == "by depth" and nj <= 32))
    every = {(product, operands, kernel, parts, narrow) for product in lp.PRODUCTS for operands in ("f32", "direct", "any")
             for kernel in lp.KERNELS for parts in (False, True) for narrow in (False, True) if kernel == "by depth" or not narrow}
    assert covered == every, every ^ covered
    assert lp.plans(exe, [("input_grad", "bf16", 700000, 256, 4096)])[0][0] == "large"         # the long tensors' product
