"""CPU-only checks of the rule that gives each product of 8-bit rows its kernel."""
import random

import pytest

from tests import int8_plan as ip

pytestmark = pytest.mark.skipif(ip.compiler() is None, reason="no C++ compiler")
TILE = {"token": (2, 1), "few 16": (16, 16), "few 32": (16, 32), "64": (64, 64), "128": (128, 128), "256": (256, 256)}
THREADS = {"token": 256, "few 16": 512, "few 32": 512, "64": 256, "128": 512, "256": 512}


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return ip.build(tmp_path_factory.mktemp("int8_plan"))


def _check(asked, p):
    """A plan that covers its output and depth, that one launch holds, and whose parts fit the workspace."""
    m, n, k = asked
    kernel, deep, parts, ti, tj, codes, us = p
    bi, bj = TILE[kernel]
    stride = -(-k // 32) * 32
    assert us >= 0, (asked, p)
    assert (ti - 1) * bi < n <= ti * bi and (tj - 1) * bj < m <= tj * bj, (asked, p)
    assert (parts - 1) * codes < stride <= parts * codes and codes % 128 == 0, (asked, p)
    groups = (ti + 7) // 8 * 8 * tj if kernel.startswith("few") else ti * tj * parts
    assert groups * THREADS[kernel] < 1 << 32, (asked, p)
    assert kernel in ("64", "128", "256") or (parts == 1 and not deep)
    if parts > 1:
        assert ti * tj <= 8192 and ti * tj * parts * bi * bj * 4 <= 64 << 20, (asked, p)
    assert (kernel == "token") == (m == 1)


def test_any_size(exe):
    """Random sizes, and the largest that the entry point takes."""
    r = random.Random(3)
    size = lambda most: int(round(most ** r.random()))  # noqa: E731
    asked = [(size(1 << 16), size(1 << 16), size(131040)) for _ in range(3000)]
    for m, n in ((1, 1 << 20), (1 << 16, 1 << 20), (1 << 20, 1 << 16), (1 << 30, 64), (1 << 30, 1), (1 << 30, 128 // 2), (2, 1 << 20)):
        asked += [(m, n, k) for k in (1, 32, 131040)]
    for a, p in zip(asked, ip.plans(exe, asked)):
        _check(a, p)


def test_cases_take_the_kernels_they_are_for(exe):
    for c, p in zip(ip.CASES, ip.plans(exe, [c[:3] for c in ip.CASES])):
        _check(c[:3], p)
        assert (p[0], p[1], p[2] > 1) == c[3:], (c, p)
    assert {c[3] for c in ip.CASES} == set(ip.KERNELS)
    assert {c[3:] for c in ip.CASES} >= {(k, d, s) for k in ("64", "128") for d, s in ((False, False), (True, False), (True, True))}


@pytest.mark.parametrize("asked,kernel", [((1, 11008, 4096), "token"), ((16, 4096, 4096), "few 16"), ((64, 11008, 4096), "64"), ((1024, 4096, 4096), "128"),
                                          ((4096, 4096, 11008), "256"), ((4096, 11008, 4096), "256")])
def test_choice(exe, asked, kernel):
    assert ip.plans(exe, [asked])[0][0] == kernel


def test_contexts_side_by_side_share_sums_in_parts(exe):
    """What tests/test_gpu_block_graphs.py multiplies."""
    assert ip.plans(exe, [(64, 2048, 11008)])[0][2] > 1
