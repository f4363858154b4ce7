"""GPU tests of every kernel that serves the linear layer's products, at sizes that take it (tests/linear_plan.py: CASES; the CPU
tests check that they do), with the sum whole and in parts, against products in float64.

Tolerances: those of tests/test_gpu_linear.py (sums: u S (8 + 4 sqrt(n)) of n terms whose magnitudes add up to S; gelu and silu: 5e-7 (1 + |z|);
outputs rounded once).  Inputs lie in frames of NaN: rows 8 elements apart where they go straight into LDS, 5 and off by 3 else."""
import math

import pytest

from paper_2506_17974_amd import binding as B
from tests import linear_plan as lp
from tests.test_gpu_linear import HALF_ULP, U, _frame, _say, _t, _untouched, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
KINDS = [c[:1] + (kind,) + c[1:] for c in lp.CASES for kind in (("f32",) if c[1] == "f32" else ("bf16", "f16"))]


def _cases(product):
    return pytest.mark.parametrize("kind,operands,m,n,k,kernel,parts", [c[1:] for c in KINDS if c[0] == product])


def _random(shape, kind, frame, seed, scale=1.0):
    """Normal values in a frame of NaN, and the same in float64."""
    import torch
    v, _ = _frame(shape, kind, float("nan"), *frame)
    v.copy_(torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale)
    return v, v.double()


def _close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d beyond the bound, worst %g of it" % (what, bad.sum(), bad.numel(),
                                                                           ((got.double() - want).abs() / tol)[bad].max())


def _rounded(kind, size):
    rel, absolute = HALF_ULP[kind]
    return rel * size + absolute


def _bound(a, b, n):
    return U * (a.abs() @ b.abs()) * (8 + 4 * n ** 0.5)


def _activated(z, act):
    import torch
    if act == "gelu":
        return z * torch.special.erfc(z / -math.sqrt(2)) / 2
    return {"none": z, "relu": z.clamp(min=0), "silu": z * torch.sigmoid(z)}[act]


def _check_kept(held, z, dz, kind):
    """A checkpoint of values that are known to +-dz: codes within half a step, exponents of a value within the bound."""
    import torch
    n = z.shape[1]
    low, high = {"f16": (-24, 9)}.get(kind, (-126, 121))
    assert not held.codes[:, n:].any()
    e = held.exponents.double() - 127
    assert (e >= low).all() and (e <= high).all()
    unit = torch.exp2(e).repeat_interleave(32, 1)[:, :n]
    assert ((held.codes[:, :n].double() * unit - z).abs() <= 0.5 * unit + dz).all()
    of_group = lambda v: torch.nn.functional.pad(v, (0, -n % 32)).view(len(v), -1, 32).amax(-1)
    assert ((of_group(z.abs() - dz) < 127.5 * torch.exp2(e)) | (e == high)).all()
    assert ((of_group(z.abs() + dz) >= 127.5 * torch.exp2(e - 1)) | (e == low)).all()


def _frames(operands):
    return (8, 8) if operands == "direct" else (5, 3)


@_cases("forward")
def test_forward(ops, kind, operands, m, n, k, kernel, parts):
    import torch
    _say("forward", kind, operands, m, n, k, kernel, parts)
    frame = _frames(operands)
    x, xv = _random((m, k), kind, frame, 1)
    w, wv = _random((n, k), kind, frame, 2, k ** -0.5)
    b, bv = _random((1, n), kind, (0, frame[1]), 3)
    r, rv = _random((m, n), kind, frame, 4)
    size = _bound(xv, wv.t().contiguous(), k)
    z0 = xv @ wv.t().contiguous()
    for act, bias, residual, keep in (("gelu", True, True, True), ("silu", True, False, True), ("none", False, False, False), ("relu", False, True, True)):
        out, flat = _frame((m, n), kind, 55.0, *frame)
        kept = [B.Checkpoint.empty(m, n), B.Checkpoint.empty(m, n)] if keep else [None, None]
        for c in kept:
            if c:
                c.codes.fill_(99)
        call = lambda **o: ops.forward(x, w, b[0] if bias else None, r if residual else None, act=act, **o)
        call(out=out, save_z=kept[0], save_y=kept[1])
        assert _untouched(flat, out, 55.0)
        z = z0 + bv if bias else z0
        y = _activated(z, act) + (rv if residual else 0)
        dz = size + 2 * U * z.abs()
        dy = (1.13 if act != "none" else 1.0) * dz + (5e-7 * (1 + z.abs()) if act in ("gelu", "silu") else 0) + 4 * U * y.abs()
        _close(out, y, dy + _rounded(kind, y.abs() + dy), act)
        if keep:
            _check_kept(kept[0], z, dz, kind)
            same = ops.save(out)
            assert torch.equal(same.codes, kept[1].codes) and torch.equal(same.exponents, kept[1].exponents)
        assert torch.equal(call(), out)                         # and the same bits again


@_cases("input_grad")
def test_input_grad(ops, kind, operands, m, n, k, kernel, parts):
    import torch
    _say("input grad", kind, operands, m, n, k, kernel, parts)
    frame = _frames(operands)
    dz, dzv = _random((m, n), kind, frame, 5)
    w, wv = _random((n, k), kind, frame, 6, n ** -0.5)
    out, flat = _frame((m, k), kind, 55.0, *frame)
    ops.input_grad(dz, w, out=out)
    assert _untouched(flat, out, 55.0)
    want, tol = dzv @ wv, _bound(dzv, wv, n)
    _close(out, want, tol + _rounded(kind, want.abs() + tol), "dx")
    assert torch.equal(ops.input_grad(dz, w), out)


@_cases("weight_grad")
def test_weight_grad(ops, kind, operands, m, n, k, kernel, parts):
    import torch
    _say("weight grad", kind, operands, m, n, k, kernel, parts)
    frame = _frames(operands)
    x, _ = _random((m, k), kind, frame, 7)
    held = ops.save(x)
    hv = ops.load(held, torch.float32).double()
    dz, dzv = _random((m, n), kind, frame, 8, 1e-2)
    want, tol = dzv.t().contiguous() @ hv, _bound(dzv.t().contiguous(), hv, m)
    for grad in ("f32", "bf16"):
        out, flat = _frame((n, k), grad, 55.0, 5, 3)
        ops.weight_grad(dz, held, out=out)
        assert _untouched(flat, out, 55.0)
        _close(out, want, tol + _rounded(grad, want.abs() + tol), "dw")
        assert torch.equal(ops.weight_grad(dz, held, dtype=_t(grad)), out)
        before = out.double()
        ops.weight_grad(dz, held, out=out, accumulate=True)
        assert _untouched(flat, out, 55.0)
        more = before.abs() + want.abs()
        _close(out, before + want, tol + 2 * U * more + _rounded(grad, more + tol), "dw added")


def test_long_tensors_through_the_large_kernel(ops):
    """Offsets that pass 32 bits in a product of whole tiles: what is at the end of long tensors, and that nothing is where dz is 0."""
    import torch
    _say("long tensors, large kernel")
    m, k, n, tail = 700000, 4096, 256, 1000                 # 5.3 GiB of bfloat16
    gen = torch.Generator(device="cuda").manual_seed(4)
    dz = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
    dz[-tail:] = torch.randn((tail, n), generator=gen, device="cuda")
    w = (torch.randn((n, k), generator=gen, device="cuda") / 16).to(torch.bfloat16)
    dx = ops.input_grad(dz, w)
    assert not dx[:-tail].any()
    d, wv = dz[-tail:].double(), w.double()
    want, tol = d @ wv, _bound(d, wv, n)
    _close(dx[-tail:], want, tol + _rounded("bf16", want.abs() + tol), "dx")
    codes = torch.zeros((m, k), dtype=torch.int8, device="cuda")
    codes[-tail:] = torch.randint(-127, 128, (tail, k), generator=gen, device="cuda", dtype=torch.int8)
    held = B.Checkpoint(codes, torch.full((m, k // 32), 121, dtype=torch.uint8, device="cuda"), k)
    z = ops.load(B.Checkpoint(codes[-tail:], held.exponents[-tail:], k), torch.float32).double()
    g = dx[-tail:].double() * (z > 0)
    _, db = ops.activation_backward(dx, held, "relu", dz=dx)
    assert not dx[:-tail].any() and torch.equal(dx[-tail:].double(), g)
    _close(db, g.sum(0), U * g.abs().sum(0) * (8 + 4 * tail ** 0.5), "dbias")
