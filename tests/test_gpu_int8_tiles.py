"""GPU tests of every kernel of the product of 8-bit rows, at sizes that the rule gives to each (tests/test_int8_plan.py asserts that it does)."""
import pytest

from paper_2506_17974_amd import binding as B
from tests import int8_plan as ip
from tests.test_gpu_linear import U, _say, _t, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _codes(gen, m, k):
    """Codes from -128 on, zeros behind the last column."""
    import torch
    c = torch.randint(-128, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
    wide = torch.zeros((m, -(-k // 32) * 32), dtype=torch.int8, device="cuda")
    wide[:, :k] = c
    return c, wide


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", ip.CASES, ids=lambda c: "%dx%dx%d" % c[:3])
def test_every_kernel(ops, kind, case):
    """Against float64, whose sums of these integers are exact: 4 u of the product, u of the sum with the residual, and the output's rounding.  Twice, the
    second time with bias and activation off, onto the residual itself."""
    import torch
    m, n, k = case[:3]
    _say("int8 kernels", kind, *case)
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    (xc, xw), (wc, ww) = _codes(g, m, k), _codes(g, n, k)
    xs, ws = (torch.rand(s, generator=g, device="cuda") * 1e-2 + 1e-3 for s in (m, n))
    bias = torch.randn(n, generator=g, device="cuda").to(_t(kind))
    wide = torch.full((m, n + 3), float("nan"), device="cuda", dtype=_t(kind))
    residual = wide[:, 1:n + 1]
    residual.copy_(torch.randn((m, n), generator=g, device="cuda"))
    x, w = B.RowCodes(xw, xs, k), B.RowCodes(ww, ws, k)
    y = ops.int8_forward(x, w, bias, residual, act="relu")
    p = torch.matmul(xc.double(), wc.double().t().contiguous()) * (xs.double()[:, None] * ws.double())
    before = residual.double()
    for got, z in ((y, (p + bias.double()).clamp(min=0)), (None, p)):
        if got is None:
            got = ops.int8_forward(x, w, None, residual, out=residual)
        want = z + before
        tol = 5 * U * p.abs() + U * (bias.double().abs() + want.abs()) + HALF[kind] * want.abs() + (2.0 ** -25 if kind == "f16" else 0)
        bad = ~((got.double() - want).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    assert torch.isnan(wide[:, 0]).all() and torch.isnan(wide[:, n + 1:]).all()
