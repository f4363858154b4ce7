"""GPU tests of the activations' slopes and values against their formulas in float64, relative to their own size: also where they go to
0, and alike for few samples (slopes by formula) and for many (slopes from a table).

Tolerances (u = 2^-24; hardware exp2 and reciprocal are good to one unit in the last place, 2 u):
  silu  s = 1 / (1 + exp(|z|)): the exponent's argument is off by u |z|, exp, the sum and the reciprocal by 5 u, so s by (|z| + 5) u of itself;
        s (1 + z (1 - s)) by that twice (s enters twice) and 4 u more, of s (1 + |z|): under (2 |z| + 16) u s (1 + |z|).  act'(|z|) = 1 - act'(-|z|)
        is rounded once more, 2 u.
  gelu  Phi(-|z|) = t P(t) exp(-z^2 / 2) / 2: the exponent's argument is rounded three times, 1.5 z^2 u of the result, exp 2 u; t is off by 4 u and
        t P(t) reacts to that 2.5-fold at most, 10 u; the sum P 4 u, its coefficients and its fit 2 u, products 2 u: (1.5 z^2 + 20) u of itself.
        |z| phi(z): (1.5 z^2 + 5) u of itself.  1 less either is rounded once more, 2 u; z Phi(z) by another 2 u.
  dz    one more product, 2 u; outputs are rounded to their type; what is below the normal numbers may be 0.
"""
import math

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


def _gelu_slope(z):
    import torch
    a = z.abs()
    phi, tail = torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi), 0.5 * torch.special.erfc(a / math.sqrt(2))
    a_phi = torch.where(phi > 0, a * phi, phi)
    s = tail - a_phi
    square = torch.clamp(a * a, max=1e4)                     # beyond, all of it is 0
    return torch.where(z < 0, s, 1 - s), U * ((1.5 * square + 20) * tail + (1.5 * square + 5) * a_phi) + torch.where(z < 0, 0.0, 2 * U) + a.clamp(max=20) * 2.0 ** -126


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
    _slopes(ops, kind, samples, features, low, high, "silu", _silu_slope)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", [(100, 1000), (2100, 11009), (700, 33000)])
@pytest.mark.parametrize("low,high", [(-8, -3), (-60, 30), (-126, 121)])
def test_gelu_slopes(ops, kind, samples, features, low, high):
    _slopes(ops, kind, samples, features, low, high, "gelu", _gelu_slope)


def _slopes(ops, kind, samples, features, low, high, act, slope):
    import torch
    _say(act, "slopes", kind, samples, features, low, high)
    held, z = _codes(samples, features, low, high, 3)
    dy = torch.randn((samples, features), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(_t(kind))
    dz, _ = ops.activation_backward(dy, held, act)
    _check(kind, dz, dy, *slope(z))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples", [1, 70, 1000])
def test_gelu_values(ops, kind, samples):
    """gelu(x I^T): z is x itself, whose last place decides what its tail can be held to."""
    import torch
    _say("gelu values", kind, samples)
    n = 320
    z = torch.linspace(-14, 14, samples * n, device="cuda", dtype=torch.float64).to(_t(kind)).view(samples, n)
    y = ops.forward(z, torch.eye(n, device="cuda", dtype=_t(kind)), act="gelu").double()
    x = z.double()
    tail = 0.5 * torch.special.erfc(x.abs() / math.sqrt(2))
    want = x * torch.where(x < 0, tail, 1 - tail)
    tol = x.abs() * (U * (1.5 * x * x + 20) * tail + torch.where(x < 0, 0.0, U)) + 2 * U * want.abs()
    rel, absolute = HALF_ULP[kind]
    tol = tol + rel * (want.abs() + tol) + absolute + 2.0 ** -126
    bad = ~((y - want).abs() <= tol)
    assert not bad.any(), "%d beyond the bound, e.g. %s for %s" % (bad.sum(), y[bad][:4].tolist(), want[bad][:4].tolist())
