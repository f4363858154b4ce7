"""GPU tests of the activations' slopes and values against their formulas in float64, relative to their own size: also where they go to
0, and alike for few samples (slopes by formula) and for many (slopes from a table).

Tolerances (u = 2^-24; hardware exp2 and reciprocal are good to one unit in the last place, 2 u):
  silu  s = 1 / (1 + exp(|z|)): the exponent's argument is off by u |z|, exp, the sum and the reciprocal by 5 u, so s by (|z| + 5) u of itself;
        s (1 + z (1 - s)) by that twice (s enters twice) and 4 u more, of s (1 + |z|): under (2 |z| + 16) u s (1 + |z|).  act'(|z|) = 1 - act'(-|z|)
        is rounded once more, 2 u.
  dz    one more product, 2 u; outputs are rounded to their type; what is below the normal numbers may be 0.
"""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import HALF_ULP, TYPES, U, _say, _t, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu


def _codes(samples, features, low, high, seed):
    """A checkpoint of every code at exponents from low to high, a NaN group among them, and what it stands for in float64."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    groups = -(-features // 32)
    codes = torch.randint(-127, 128, (samples, groups * 32), generator=g, device="cuda", dtype=torch.int8)
    codes[:, features:] = 0
    exps = torch.randint(low + 127, high + 128, (samples, groups), generator=g, device="cuda").to(torch.uint8)
    exps[samples // 2, groups // 2] = 255
    unit = torch.exp2(exps.double() - 127)
    unit[exps == 255] = float("nan")
    z = (codes.double().view(samples, groups, 32) * unit[:, :, None]).view(samples, -1)[:, :features]
    return B.Checkpoint(codes, exps, features), z


def _silu_slope(z):
    """act'(z) and the bound of its error."""
    import torch
    s, a = torch.sigmoid(-z.abs()), z.abs()
    tail = s * (1 - a * (1 - s))
    return torch.where(z < 0, tail, 1 - tail), U * s * (1 + a) * (2 * a + 16) + torch.where(z < 0, 0.0, 2 * U)


def _check(kind, got, dy, slope, bound):
    rel, absolute = HALF_ULP[kind]
    want = dy.double() * slope
    tol = dy.double().abs() * bound + 2 * U * want.abs()
    tol = tol + rel * (want.abs() + tol) + absolute + 2.0 ** -126
    bad = ~((got.double() - want).abs() <= tol) & ~slope.isnan()
    assert not bad.any(), "%d beyond the bound, e.g. %s for %s" % (bad.sum(), got[bad][:4].tolist(), want[bad][:4].tolist())
    assert got[slope.isnan()].isnan().all()


# From 2.1e7 values on (three rounds of 1280 workgroups) slopes come from the table.
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", [(100, 1000), (2100, 11009), (700, 33000)])
@pytest.mark.parametrize("low,high", [(-8, 1), (-60, 30), (-126, 121)])
def test_silu_slopes(ops, kind, samples, features, low, high):
    import torch
    _say("silu slopes", kind, samples, features, low, high)
    held, z = _codes(samples, features, low, high, 3)
    dy = torch.randn((samples, features), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(_t(kind))
    dz, _ = ops.activation_backward(dy, held, "silu")
    _check(kind, dz, dy, *_silu_slope(z))
