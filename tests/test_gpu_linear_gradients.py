"""GPU tests of the linear layer's gradients against central differences of its forward pass, along directions in which the terms add up
instead of cancelling, so that a gradient of 0 or a slope of 1 is far outside of the bound."""
import math

import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import U, _say, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
# largest second and third derivative: gelu phi (2 - z^2) and phi z (z^2 - 4), silu s' (2 + z (1 - 2 s)) and what follows; relu: none off its kink
CURVES = {"none": (0.0, 0.0), "relu": (0.0, 0.0), "gelu": (0.8, 0.8), "silu": (0.5, 0.5)}


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("direction", ["x", "w", "b"])
def test_differences_that_add_up(ops, act, direction):
    """sum of c y along a direction that moves z by u: c = |c| sign(u), but 0 where relu's kink is within reach.  Bound: the differences' own
    h^2 / 6 of the third derivative, the second derivative times what the checkpoint has z off by, and the forward pass's fp32
    errors over 2 h."""
    import torch
    _say("differences that add up", act, direction)
    g = torch.Generator(device="cuda").manual_seed(17)
    m, n, k, h = 48, 40, 64, 2.0 ** -6
    x = torch.randint(-60, 61, (m, k), generator=g, device="cuda").float().mul(2.0 ** -6)
    x[:, ::32] = 1.25                                   # every group has the exponent -6: x is its own checkpoint
    w = torch.randn((n, k), generator=g, device="cuda") / 16
    b = torch.randn(n, generator=g, device="cuda") / 4
    d = {"x": torch.randn((m, k), generator=g, device="cuda"), "w": torch.randn((n, k), generator=g, device="cuda") / 16,
         "b": torch.randn(n, generator=g, device="cuda")}[direction]
    held, zk = ops.save(x), B.Checkpoint.empty(m, n)
    assert torch.equal(ops.load(held, torch.float32), x)
    ops.forward(x, w, b, act=act, save_z=zk)
    z = x.double() @ w.double().t().contiguous() + b.double()
    off = (ops.load(zk, torch.float32).double() - z).abs()
    u = {"x": lambda: d.double() @ w.double().t().contiguous(), "w": lambda: x.double() @ d.double().t().contiguous(),
         "b": lambda: d.double().expand(m, n)}[direction]()
    c = torch.randn((m, n), generator=g, device="cuda").abs() * u.sign().float()
    if act == "relu":
        c[z.abs() <= 1.01 * h * u.abs() + off] = 0
    dz, db = ops.activation_backward(c, zk, act)
    grad = {"x": lambda: ops.input_grad(dz, w), "w": lambda: ops.weight_grad(dz, held), "b": lambda: db}[direction]()
    at = lambda s: ops.forward(x + s * d if direction == "x" else x, w + s * d if direction == "w" else w, b + s * d if direction == "b" else b, act=act)
    # the moved operands are rounded: to what fp32 makes of them the differences are exact up to u of their size
    want = ((at(h).double() - at(-h).double()) / (2 * h) * c.double()).sum().item()
    got = (grad.double() * d.double()).sum().item()
    second, third = CURVES[act]
    size = x.double().abs() @ w.double().abs().t().contiguous() + b.double().abs() + h * u.abs()
    forward = 1.13 * U * size * (10 + 4 * math.sqrt(k)) + 5e-7 * (1 + z.abs()) + 6 * U * (1 + z.abs())
    mag = c.double().abs()
    tol = (mag * (u.abs().pow(3) * third * h * h / 6 + u.abs() * off * second + forward / h)).sum().item()
    tol += (mag * u.abs()).sum().item() * 1.13 * U * (16 + 8 * math.sqrt(k + m))        # the gradient's own sums
    assert want > 20 * tol, (want, tol)                 # neither 0 nor, for an activation, a slope of 1 would pass
    if act != "none":
        assert (mag * u.abs()).sum().item() - want > 20 * tol
    assert abs(want - got) <= tol, (want, got, tol)
