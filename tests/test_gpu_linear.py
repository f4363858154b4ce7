"""GPU tests of the linear layer (include/lqsgd_linear.h) against oracle/linear_oracle.py in float64.

Tolerances, from the arithmetic (u = 2^-24, S = the sum of the magnitudes that an output adds up, n = how many):
  sums in fp32      |error| <= u S (8 + 4 sqrt(n)): each of n additions rounds a partial sum that is at most S, independently (6
                    standard deviations are 3.5 sqrt(n)); the 8 covers the terms that the three-part split of fp32 operands
                    leaves out (under 4 u of each product) and the epilogue's own roundings
  activations       5e-7 (1 + |z|) beside: the 1.5e-7 of the rational form of Phi, and hardware exp2 and reciprocal of one ulp
  outputs           rounded once: half an ulp of the type (2^-24, 2^-8, 2^-11 relative; f16 2^-25 absolute below its normal range)
  checkpoints       exact, or within half a step of a value that is itself known to the bound above
"""
import numpy as np
import pytest

import oracle.linear_oracle as lo
from paper_2506_17974_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}
TYPES = ("f32", "bf16", "f16")


def _t(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


@pytest.fixture(scope="module")
def ops():
    o = B.LinearOps()
    yield o
    o.close()


def _say(*a):
    print("case:", *a, flush=True)


def _frame(shape, kind, fill, pad=0, offset=0):
    """A matrix inside a larger buffer full of `fill`: rows `pad` elements apart from each other, the first at `offset`."""
    import torch
    m, n = shape
    flat = torch.full((offset + m * (n + pad) + 64,), fill, dtype=_t(kind), device="cuda")
    return flat[offset:offset + m * (n + pad)].view(m, n + pad)[:, :n], flat


def _put(a, kind, pad=0, offset=0):
    """Input values with NaN around them: whatever is read beyond a row would show."""
    import torch
    v, _ = _frame(a.shape, kind, float("nan"), pad, offset)
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return v, v.double().cpu().numpy()


def _untouched(flat, view, fill):
    """Nothing outside of the view was written."""
    mark = flat.clone()
    mark[view.storage_offset():].as_strided(view.shape, view.stride()).fill_(fill)
    return bool((mark == fill).all())


def _rounded(kind, want):
    rel, absolute = HALF_ULP[kind]
    return rel * np.abs(want) + absolute


def _close(got, want, tol, what):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d beyond the bound, worst %g of it" % (what, bad.sum(), bad.size, (np.abs(got - want) / tol)[bad].max())


def _sum_bound(a, b, n):
    return U * (np.abs(a) @ np.abs(b)) * (8 + 4 * np.sqrt(n))


def _held(codes, exps, features, device="cuda"):
    import torch
    return B.Checkpoint(torch.from_numpy(codes).to(device), torch.from_numpy(exps).to(device), features)


def _host(c):
    return c.codes.cpu().numpy(), c.exponents.cpu().numpy()


def _check_kept(c, z, dz, kind):
    """A checkpoint of values that are known to +-dz."""
    codes, exps = _host(c)
    n = z.shape[1]
    assert (codes[:, n:] == 0).all()
    step = 2.0 ** (np.repeat(exps, 32, 1)[:, :n].astype(float) - 127)
    got = lo.load(codes, exps, n)
    assert (np.abs(got - z) <= 0.5 * step + dz).all()
    # the exponent is the one of some value within the bound
    big, lohi = np.abs(z) + dz, lo.BOUNDS[kind]
    for g in range(exps.shape[1]):
        s = slice(32 * g, min(n, 32 * g + 32))
        e = exps[:, g].astype(int) - 127
        assert (e >= lohi[0]).all() and (e <= lohi[1]).all()
        top = big[:, s].max(1)
        least = (np.abs(z) - dz)[:, s].max(1)
        assert ((least < 127.5 * 2.0 ** e) | (e == lohi[1])).all()
        assert ((top >= 127.5 * 2.0 ** (e - 1)) | (e == lohi[0])).all()


# (samples, rows, cols): single values, single tokens, edges of groups and tiles, sizes of the benchmark's layers, long sums
SHAPES = [(1, 1, 1), (1, 10, 512), (1, 257, 1155), (2, 64, 27), (3, 5, 7), (4, 1000, 2049), (5, 33, 65), (7, 129, 131), (13, 64, 800),
          (16, 96, 256), (17, 32, 25), (31, 31, 33), (33, 65, 33), (64, 1024, 96), (65, 10, 1024), (127, 128, 127), (129, 127, 64),
          (255, 256, 257), (256, 257, 255), (300, 257, 513), (511, 40, 8), (640, 384, 320), (1000, 16, 16), (33, 200, 4096), (96, 4096, 40)]
LONG = [(9000, 10, 33), (5, 10, 11008), (40, 9000, 24), (2500, 64, 64)]


# ---------------------------------------------------------------------------
# checkpoints
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features,pad,offset", [(1, 1, 0, 0), (1, 31, 0, 0), (3, 32, 0, 0), (2, 33, 1, 1), (17, 65, 0, 3), (5, 1155, 5, 0),
                                                         (300, 27, 0, 0), (64, 4096, 0, 0), (33, 513, 7, 8), (1000, 8, 0, 0)])
def test_save_and_load(ops, kind, samples, features, pad, offset):
    import torch
    _say("save", kind, samples, features, pad, offset)
    rng = np.random.default_rng(samples * 1000 + features)
    a = rng.standard_normal((samples, features)) * np.exp(2 * rng.standard_normal((samples, 1)))
    if features > 30:
        a[0, :32] = 0                                              # an empty group
        a[-1, 3] = 127.5 / 64                                      # may be on the boundary of its exponent
    x, v = _put(a.astype(np.float32), kind, pad, offset)
    c = ops.save(x)
    want = lo.save(v, kind)
    codes, exps = _host(c)
    assert np.array_equal(exps, want[1]) and np.array_equal(codes, want[0])
    back = lo.load(*want, features)
    for out_kind in {kind, "f32"}:
        out, flat = _frame((samples, features), out_kind, 77.0, pad, offset)
        ops.load(c, out=out)
        assert np.array_equal(out.double().cpu().numpy(), back)    # exact in its own type and in a wider one
        assert _untouched(flat, out, 77.0)
    assert torch.equal(ops.load(c, _t(kind)).float(), ops.load(c, torch.float32))


@pytest.mark.parametrize("kind", TYPES)
def test_checkpoints_of_extreme_values(ops, kind):
    _say("extremes", kind)
    top = {"f32": 3.4028234e38, "bf16": 3.3895e38, "f16": 65504.0}[kind]
    low = {"f32": 1e-45, "bf16": 1e-40, "f16": 6e-8}[kind]
    a = np.zeros((8, 64), np.float32)
    a[0, 1], a[0, 40] = top, -top
    a[1, 5], a[1, 33] = low, -low
    a[2, 7] = np.inf
    a[3, 9] = np.nan
    a[4, 50] = -np.inf
    a[5, :] = np.float32(top) * np.linspace(-1, 1, 64, dtype=np.float32)
    a[6, :] = 1e-37 if kind != "f16" else 3e-7
    a[7, :] = -0.0
    x, v = _put(a, kind)
    c = ops.save(x)
    want = lo.save(v, kind)
    codes, exps = _host(c)
    assert np.array_equal(exps, want[1]) and np.array_equal(codes, want[0])
    out = ops.load(c, _t(kind)).double().cpu().numpy()
    back = lo.load(codes, exps, 64)
    assert np.array_equal(np.isnan(out), np.isnan(back)) and np.isnan(out).sum() == 96
    assert np.array_equal(out[~np.isnan(out)], back[~np.isnan(back)]) and np.isfinite(out[~np.isnan(out)]).all()


# ---------------------------------------------------------------------------
# forward
# ---------------------------------------------------------------------------
def _forward(ops, kind, shape, act, bias, residual, keep, pad=0, offset=0, seed=0):
    m, n, k = shape
    rng = np.random.default_rng(1000 * m + 10 * n + k + seed)
    x, xv = _put(rng.standard_normal((m, k)), kind, pad, offset)
    w, wv = _put(rng.standard_normal((n, k)) / np.sqrt(k), kind, 3 * pad, offset)
    b = bv = r = rv = None
    if bias:
        b, bv = _put(rng.standard_normal((1, n)), kind, 0, offset)
        b, bv = b[0], bv[0]
    if residual:
        r, rv = _put(rng.standard_normal((m, n)), kind, pad, offset)
    out, flat = _frame((m, n), kind, 55.0, pad, offset)
    zk, yk = (B.Checkpoint.empty(m, n), B.Checkpoint.empty(m, n)) if keep else (None, None)
    if keep:
        zk.codes.fill_(99), yk.codes.fill_(99)
    y = ops.forward(x, w, b, r, act=act, out=out, save_z=zk, save_y=yk)
    assert y is out and _untouched(flat, out, 55.0)
    z64, y64 = lo.forward(xv, wv, bv, rv, act)
    dz = _sum_bound(xv, wv.T, k) + U * 2 * np.abs(z64)
    dy = (1.13 if act != "none" else 1.0) * dz + (5e-7 * (1 + np.abs(z64)) if act in ("gelu", "silu") else 0) + 4 * U * np.abs(y64)
    _close(out, y64, dy + _rounded(kind, np.abs(y64) + dy), "y")
    if keep:
        _check_kept(zk, z64, dz, kind)
        same = ops.save(out)
        assert np.array_equal(_host(same)[0], _host(yk)[0]) and np.array_equal(_host(same)[1], _host(yk)[1])
    return out


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_forward(ops, kind, shape):
    _say("forward", kind, shape)
    i = SHAPES.index(shape) if shape in SHAPES else 2
    _forward(ops, kind, shape, ("none", "relu", "gelu", "silu")[i % 4], i % 2 == 0, i % 3 == 0, keep=i % 2 == 1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(1, 70, 64), (40, 70, 96), (200, 160, 128)])
def test_forward_epilogues(ops, kind, act, shape):
    _say("epilogue", kind, act, shape)
    for bias in (False, True):
        for residual in (False, True):
            _forward(ops, kind, shape, act, bias, residual, keep=bias != residual)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape,pad,offset", [((1, 65, 40), 3, 1), ((18, 33, 64), 8, 0), ((70, 130, 72), 1, 0), ((130, 70, 264), 16, 8), ((130, 258, 100), 5, 3)])
def test_forward_strides(ops, kind, shape, pad, offset):
    _say("strides", kind, shape, pad, offset)
    _forward(ops, kind, shape, "gelu", True, True, True, pad, offset)


@pytest.mark.parametrize("kind", TYPES)
def test_forward_onto_the_residual(ops, kind):
    _say("in place", kind)
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    for m, n, k in ((3, 100, 50), (300, 200, 64), (40, 64, 4000)):
        x, w, r = (torch.randn(s, generator=g, device="cuda").to(_t(kind)) for s in ((m, k), (n, k), (m, n)))
        want = ops.forward(x, w, None, r, act="silu")
        got = ops.forward(x, w, None, r, act="silu", out=r)
        assert got is r and torch.equal(got, want)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", [(5, 40, 70), (70, 40, 96), (300, 300, 130)])
def test_forward_of_values_that_are_not_finite(ops, kind, shape):
    """A NaN in a sample reaches that sample alone, one in a weight its feature alone; an infinity what the formula says, in the
    16-bit types, and something that is not finite in fp32."""
    import torch
    _say("not finite", kind, shape)
    m, n, k = shape
    g = torch.Generator(device="cuda").manual_seed(9)
    for bad in (float("nan"), float("inf")):
        x = torch.randn((m, k), generator=g, device="cuda").to(_t(kind))
        w = torch.rand((n, k), generator=g, device="cuda").add(0.1).to(_t(kind))
        clean = ops.forward(x, w)
        x[3, k - 1] = bad
        zk = B.Checkpoint.empty(m, n)
        y = ops.forward(x, w, act="relu", save_z=zk)
        rest = torch.arange(m, device="cuda") != 3
        assert not torch.isfinite(y[3]).any() and torch.equal(y[rest], clean[rest].clamp(min=0))
        if kind != "f32":
            assert (y[3].isnan() if bad != bad else y[3] == bad).all()
        assert (zk.exponents[3] == 255).all() and (zk.exponents[rest] != 255).all()
        assert ops.load(zk)[3].isnan().all()
        x[3, k - 1] = 0
        w[7, 0] = bad
        y = ops.forward(x, w)
        rest = torch.arange(n, device="cuda") != 7
        assert not torch.isfinite(y[:, 7]).any() and torch.isfinite(y[:, rest]).all()


@pytest.mark.parametrize("scale_x,scale_w", [(3.4e38, 1e-30), (1e-30, 1e30), (2.0 ** -112, 1e30), (2.0 ** -130, 1e35)])
def test_fp32_operands_of_any_size(ops, scale_x, scale_w):
    """The three terms of an fp32 operand reach from the largest numbers to multiples of 2^-133."""
    _say("sizes", scale_x, scale_w)
    rng = np.random.default_rng(23)
    x, xv = _put((rng.random((70, 96)) * 0.5 + 0.5) * scale_x, "f32")
    w, wv = _put(rng.standard_normal((80, 96)) * scale_w, "f32")
    want = xv @ wv.T
    tol = _sum_bound(xv, wv.T, 96) + 2.0 ** -133 * np.abs(wv).sum(1) + HALF_ULP["f32"][0] * np.abs(want)
    _close(ops.forward(x, w), want, tol, "y")
    _close(ops.input_grad(x, w.t().contiguous()), want, tol, "dx")


# ---------------------------------------------------------------------------
# backward
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_input_grad(ops, kind, shape):
    _say("input grad", kind, shape)
    m, n, k = shape
    rng = np.random.default_rng(m + n + k)
    for pad, offset in ((0, 0), (5, 1)):
        dz, dzv = _put(rng.standard_normal((m, n)), kind, pad, offset)
        w, wv = _put(rng.standard_normal((n, k)) / np.sqrt(n), kind, pad, offset)
        out, flat = _frame((m, k), kind, 55.0, pad, offset)
        ops.input_grad(dz, w, out=out)
        assert _untouched(flat, out, 55.0)
        want, tol = lo.input_grad(dzv, wv), _sum_bound(dzv, wv, n)
        _close(out, want, tol + _rounded(kind, np.abs(want) + tol), "dx")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_weight_grad(ops, kind, shape):
    import torch
    _say("weight grad", kind, shape)
    m, n, k = shape
    rng = np.random.default_rng(m + n + 7 * k)
    xv = rng.standard_normal((m, k))
    if kind != "f32":
        xv = torch.from_numpy(xv).to(_t(kind)).double().numpy()
    codes, exps = lo.save(xv, kind)
    held, hv = _held(codes, exps, k), lo.load(codes, exps, k)
    for pad, offset, grad in ((0, 0, "f32"), (3, 1, "f32"), (0, 0, "bf16")):
        dz, dzv = _put(rng.standard_normal((m, n)) * 1e-2, kind, pad, offset)
        out, flat = _frame((n, k), grad, 55.0, pad, offset)
        ops.weight_grad(dz, held, out=out)
        assert _untouched(flat, out, 55.0)
        want, tol = lo.weight_grad(dzv, hv), _sum_bound(dzv.T, hv, m)
        _close(out, want, tol + _rounded(grad, np.abs(want) + tol), "dw")
        before = out.double().cpu().numpy()
        ops.weight_grad(dz, held, out=out, accumulate=True)
        assert _untouched(flat, out, 55.0)
        more = np.abs(before) + np.abs(want)
        _close(out, before + want, tol + 2 * U * more + _rounded(grad, more + tol), "dw added")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("samples,rows,pad", [(1, 1, 0), (1, 1000, 0), (3, 7, 1), (17, 65, 0), (64, 1024, 0), (129, 33, 5), (2000, 10, 0), (777, 513, 0),
                                              (70000, 3, 0)])
def test_activation_backward(ops, kind, act, samples, rows, pad):
    _say("activation backward", kind, act, samples, rows, pad)
    rng = np.random.default_rng(samples + rows)
    codes, exps = lo.save(rng.standard_normal((samples, rows)) * 2, kind) if samples < 5000 else (
        rng.integers(-127, 128, (samples, 32)).astype(np.int8), rng.integers(118, 124, (samples, 1)).astype(np.uint8))
    z = lo.load(codes, exps, rows)
    dy, dyv = _put(rng.standard_normal((samples, rows)), kind, pad, pad)
    dz, flat = _frame((samples, rows), kind, 55.0, pad, pad)
    held = _held(codes, exps, rows) if act != "none" else None
    _, db = ops.activation_backward(dy, held, act, dz=dz)
    assert _untouched(flat, dz, 55.0)
    want, wantb = lo.activation_backward(dyv, z, act)
    tol = np.abs(dyv) * (5e-7 * (1 + np.abs(z)) if act in ("gelu", "silu") else 0) + 4 * U * np.abs(want)
    _close(dz, want, tol + _rounded(kind, np.abs(want) + tol), "dz")
    tolb = tol.sum(0) + U * np.abs(want).sum(0) * (8 + 4 * np.sqrt(samples))
    _close(db, wantb, tolb, "dbias")
    # parts of it, in place, and added to what is there
    _, again = ops.activation_backward(dy, held, act, want_dz=False)
    assert again.equal(db)
    ops.activation_backward(dy, held, act, want_dz=False, dbias=db, accumulate=True)
    _close(db, 2 * wantb, 2 * tolb + 4 * U * np.abs(wantb), "dbias added")
    alone, none = ops.activation_backward(dy, held, act, want_dbias=False)
    assert none is None and alone.equal(dz)
    ops.activation_backward(dy, held, act, dz=dy, want_dbias=False)
    assert dy.equal(dz)


@pytest.mark.parametrize("kind", TYPES)
def test_backward_of_groups_that_are_not_finite(ops, kind):
    import torch
    _say("NaN groups", kind)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((70, 100), generator=g, device="cuda").to(_t(kind))
    dz = torch.randn((70, 40), generator=g, device="cuda").to(_t(kind))
    clean = ops.weight_grad(dz, ops.save(x))
    x[11, 33] = float("inf")
    held = ops.save(x)
    dw = ops.weight_grad(dz, held)
    assert dw[:, 32:64].isnan().all()
    rest = torch.cat([torch.arange(32), torch.arange(64, 100)]).cuda()
    assert torch.equal(dw[:, rest], clean[:, rest])
    for act in ("relu", "gelu", "silu"):
        out, db = ops.activation_backward(torch.ones_like(x), held, act)
        assert out[11, 32:64].isnan().all() and out.isnan().sum() == 32
        assert db[32:64].isnan().all() and db.isnan().sum() == 32


@pytest.mark.parametrize("kind", TYPES)
def test_no_samples(ops, kind):
    import torch
    _say("no samples", kind)
    T = _t(kind)
    x, w, dz = torch.empty((0, 40), dtype=T, device="cuda"), torch.ones((24, 40), dtype=T, device="cuda"), torch.empty((0, 24), dtype=T, device="cuda")
    c = ops.save(x)
    assert ops.load(c, T).shape == (0, 40)
    assert ops.forward(x, w, act="gelu", save_z=B.Checkpoint.empty(0, 24)).shape == (0, 24)
    assert ops.input_grad(dz, w).shape == (0, 40)
    dw = torch.full((24, 40), 5.0, device="cuda")
    ops.weight_grad(dz, c, out=dw, accumulate=True)
    assert (dw == 5).all()
    ops.weight_grad(dz, c, out=dw)
    assert (dw == 0).all()
    db = torch.full((24,), 5.0, device="cuda")
    ops.activation_backward(dz, B.Checkpoint.empty(0, 24), "relu", dbias=db, accumulate=True)
    assert (db == 5).all()
    ops.activation_backward(dz, B.Checkpoint.empty(0, 24), "relu", dbias=db)
    assert (db == 0).all()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_gradients_are_the_differences(ops, act):
    """A layer in fp32 whose inputs are on the checkpoint's grid (x^ = x): the three gradients against central differences of the
    forward kernel along a direction.  With h = 2^-6 the differences' own error is h^2 / 6 of the third derivative (under 2 for
    these activations), and z^ is within 2^-8 of z where the slope's derivative is under 1.2."""
    import torch
    _say("differences", act)
    g = torch.Generator(device="cuda").manual_seed(17)
    m, n, k = 48, 40, 64
    x = torch.randint(-60, 61, (m, k), generator=g, device="cuda").float().mul(2.0 ** -6)
    x[:, ::32] = 1.25                                   # every group has the exponent -6: x is its own checkpoint
    w = torch.randn((n, k), generator=g, device="cuda") / 16
    b = torch.randn(n, generator=g, device="cuda") / 4
    c = torch.randn((m, n), generator=g, device="cuda")
    held = ops.save(x)
    assert torch.equal(ops.load(held, torch.float32), x)
    zk = B.Checkpoint.empty(m, n)
    ops.forward(x, w, b, act=act, save_z=zk)
    dz, db = ops.activation_backward(c, zk, act)
    dx, dw = ops.input_grad(dz, w), ops.weight_grad(dz, held)
    h = 2.0 ** -6
    for name, d, grad in (("x", torch.randn((m, k), generator=g, device="cuda"), dx), ("w", torch.randn((n, k), generator=g, device="cuda") / 16, dw),
                          ("b", torch.randn(n, generator=g, device="cuda"), db)):
        move = lambda s: ops.forward(x + s * d if name == "x" else x, w + s * d if name == "w" else w, b + s * d if name == "b" else b, act=act)
        diff = (move(h).double() - move(-h).double()) / (2 * h)
        u = x.double() @ d.double().t() if name == "w" else d.double() @ w.double().t() if name == "x" else d.double().expand(m, n)
        want, got = (diff * c).sum().item(), (grad.double() * d.double()).sum().item()
        cu = c.double().abs() * u.abs()
        z = x.double() @ w.double().t() + b
        if act == "relu":                               # its kink: values that the step or the checkpoint takes across 0
            tol = (cu * (z.abs() <= h * u.abs() + 2.0 ** -6)).sum().item() + 1e-3
        else:
            tol = (c.double().abs() * u.abs().pow(3)).sum().item() * 2 * h * h / 6 + (0 if act == "none" else 1.2 * cu.sum().item() * 2.0 ** -6) + 1e-3
            if act != "none":                           # errors of z^ are independent: far below their sum of magnitudes
                tol = min(tol, 0.02 * cu.sum().item())
        assert abs(want - got) <= tol + 2e-5 * cu.sum().item(), (name, want, got, tol)


# ---------------------------------------------------------------------------
# the same bits, long tensors, graphs, refusals
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (30, 300, 2000), (600, 500, 700), (64, 64, 20000), (20000, 64, 64)])
def test_same_bits_every_time(ops, kind, m, n, k):
    import torch
    _say("same bits", kind, m, n, k)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, dz = (torch.randn(s, generator=g, device="cuda").to(_t(kind)) for s in ((m, k), (n, k), (m, n)))
    held = ops.save(x)

    def all_of_it():
        z = B.Checkpoint.empty(m, n)
        y = ops.forward(x, w, None, dz, act="gelu", save_z=z)
        d, db = ops.activation_backward(dz, z, "gelu")
        return [y, z.codes, z.exponents, d, db, ops.input_grad(dz, w), ops.weight_grad(dz, held)]

    first = all_of_it()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, all_of_it()))


def test_tensors_beyond_4_gib(ops):
    """Rows whose offsets pass 32 bits: the last samples of long tensors are what they are on their own."""
    import torch
    _say("beyond 4 GiB")
    m, k, n = 700000, 4096, 32                          # 5.3 GiB of bfloat16
    x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    x[:1000].normal_(), x[-1000:].normal_()
    x[1000:-1000] = 0
    w = torch.randn((n, k), device="cuda").to(torch.bfloat16)
    held, tail = ops.save(x), ops.save(x[-1000:])
    assert torch.equal(held.codes[-1000:], tail.codes) and torch.equal(held.exponents[-1000:], tail.exponents)
    assert not held.codes[1000:2000].any()
    y = ops.forward(x, w)
    assert torch.equal(y[-1000:], ops.forward(x[-1000:].clone(), w)) or \
        (y[-1000:].float() - ops.forward(x[-1000:].clone(), w).float()).abs().max() <= 2.0 ** -7 * y[-1000:].float().abs().max()
    assert not y[1000:-1000].any()
    back = ops.load(held, out=x)                        # over x itself, which is not needed any more
    assert torch.equal(back[-1000:], ops.load(tail))
    dz = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
    dz[-1000:].normal_()
    dw, want = ops.weight_grad(dz, held), dz[-1000:].double().t() @ ops.load(tail, torch.float32).double()
    size = dz[-1000:].double().abs().t() @ ops.load(tail, torch.float32).double().abs()
    assert ((dw.double() - want).abs() <= U * size * (8 + 4 * 1000 ** 0.5)).all()
    dx = ops.input_grad(dz, w)
    assert not dx[:-1000].any() and torch.equal(dx[-1000:], ops.input_grad(dz[-1000:].clone(), w)) or \
        (dx[-1000:].float() - ops.input_grad(dz[-1000:].clone(), w).float()).abs().max() <= 2.0 ** -7 * dx[-1000:].float().abs().max()
    _, db = ops.activation_backward(dx, held, "relu", dz=dx)
    assert torch.isfinite(db).all()


def test_in_a_graph():
    """Forward and backward recorded once and replayed between eager work; every replay equals the eager result."""
    import torch
    _say("graph")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops = B.LinearOps()
        g = torch.Generator(device="cuda").manual_seed(21)
        m, n, k = 96, 160, 2000
        x, w, dy = (torch.randn(t, generator=g, device="cuda").to(torch.bfloat16) for t in ((m, k), (n, k), (m, n)))
        bias = torch.randn(n, generator=g, device="cuda").to(torch.bfloat16)
        xk, zk = B.Checkpoint.empty(m, k), B.Checkpoint.empty(m, n)
        y, dz, dx = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x)
        db, dw = torch.empty(n, device="cuda"), torch.empty((n, k), device="cuda")

        def step():
            ops.save(x, out=xk)
            ops.forward(x, w, bias, act="gelu", out=y, save_z=zk)
            ops.activation_backward(dy, zk, "gelu", dz=dz, dbias=db)
            ops.input_grad(dz, w, out=dx)
            ops.weight_grad(dz, xk, out=dw)

        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for seed in range(4):
            x.copy_(torch.randn((m, k), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
            step()
            want = [t.clone() for t in (y, dz, db, dx, dw, xk.codes, zk.codes)]
            for t in (y, dz, db, dx, dw, xk.codes, zk.codes):
                t.zero_()
            graph.replay()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (y, dz, db, dx, dw, xk.codes, zk.codes)))
        del graph
        ops.close()


def test_refusals(ops):
    import torch
    _say("refusals")
    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)
    x, w = f(4, 8), f(6, 8)

    def refused(code, call):
        with pytest.raises(B.LqsgdError) as e:
            call()
        assert e.value.code == code, e.value

    refused(B.ESHAPE, lambda: ops.forward(x, f(6, 7)))
    refused(B.ESHAPE, lambda: ops.forward(x, w.to(torch.bfloat16)))
    refused(B.ESHAPE, lambda: ops.forward(x.double(), w.double()))
    refused(B.ESHAPE, lambda: ops.forward(x.cpu(), w))
    refused(B.ESHAPE, lambda: ops.forward(f(8, 4).t(), w))
    refused(B.ESHAPE, lambda: ops.forward(f(1, 8).expand(4, 8), w))
    refused(B.ESHAPE, lambda: ops.forward(x, w, bias=f(5)))
    refused(B.ESHAPE, lambda: ops.forward(x, w, residual=f(4, 5)))
    refused(B.ESHAPE, lambda: ops.forward(x, w, out=f(4, 7)))
    refused(B.ESHAPE, lambda: ops.forward(x[None], w))
    refused(B.EINVAL, lambda: ops.forward(x, w, act="tanh"))
    refused(B.EINVAL, lambda: ops.forward(x, w, save_z=f(4, 32)))
    refused(B.ESHAPE, lambda: ops.forward(x, w, save_z=B.Checkpoint.empty(4, 8)))
    refused(B.ESHAPE, lambda: ops.forward(x, w, save_z=B.Checkpoint.empty(3, 6)))
    refused(B.ESHAPE, lambda: ops.forward(f(4, 0), f(6, 0)))
    refused(B.EINVAL, lambda: ops.activation_backward(x, None, "relu"))
    refused(B.EINVAL, lambda: ops.activation_backward(x, None, want_dz=False, want_dbias=False))
    refused(B.EINVAL, lambda: ops.activation_backward(x, accumulate=True))
    refused(B.ESHAPE, lambda: ops.input_grad(x, w))
    refused(B.EINVAL, lambda: ops.weight_grad(x, w))
    refused(B.ESHAPE, lambda: ops.weight_grad(x, B.Checkpoint.empty(5, 8)))
    refused(B.EINVAL, lambda: ops.weight_grad(x, B.Checkpoint.empty(4, 8), accumulate=True))
    refused(B.EINVAL, lambda: ops.weight_grad(x, B.Checkpoint.empty(4, 8), dtype=torch.float16))
    refused(B.EINVAL, lambda: ops.load(x))
    c = B.Checkpoint.empty(4, 8)
    refused(B.EINVAL, lambda: ops.load(B.Checkpoint(torch.zeros(200, dtype=torch.int8, device="cuda")[1:129].view(4, 32), c.exponents, 8)))
    with torch.cuda.stream(torch.cuda.Stream()):
        refused(B.ESTATE, lambda: ops.forward(x, w))
    gone = B.LinearOps()
    gone.close()
    refused(B.ESTATE, lambda: gone.forward(x, w))
    # the C entry points themselves
    L, h = B.lib(), ops._h
    px, pw = x.data_ptr(), w.data_ptr()
    call = lambda **k: L.lqsgd_linear_forward(h, *[k.get(n, d) for n, d in (
        ("type", 0), ("act", 0), ("samples", 4), ("rows", 6), ("cols", 8), ("x", px), ("ldx", 8), ("w", pw), ("ldw", 8), ("bias", None),
        ("residual", None), ("ldr", 0), ("y", f(4, 6).data_ptr()), ("ldy", 6), ("zc", None), ("ze", None), ("yc", None), ("ye", None))])
    assert call() == B.OK
    for bad, code in ((dict(type=3), B.EINVAL), (dict(act=4), B.EINVAL), (dict(samples=-1), B.ESHAPE), (dict(samples=(1 << 30) + 1), B.ESHAPE),
                      (dict(rows=0), B.ESHAPE), (dict(cols=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), B.ESHAPE), (dict(ldx=7), B.ESHAPE),
                      (dict(ldw=(1 << 21) + 1), B.ESHAPE), (dict(ldy=5), B.ESHAPE), (dict(x=None), B.EINVAL), (dict(w=None), B.EINVAL),
                      (dict(y=None), B.EINVAL), (dict(x=px + 2), B.EINVAL), (dict(residual=px, ldr=5), B.ESHAPE), (dict(y=px, ldy=6, residual=px, ldr=8), B.EINVAL),
                      (dict(zc=c.codes.data_ptr()), B.EINVAL), (dict(zc=c.codes.data_ptr() + 8, ze=c.exponents.data_ptr()), B.EINVAL)):
        assert call(**bad) == code, bad
        assert L.lqsgd_linear_last_error(h).decode()
    # outputs over inputs
    square = f(8, 8)
    refused(B.EINVAL, lambda: ops.forward(square, f(8, 8), out=square))
    refused(B.EINVAL, lambda: ops.forward(f(8, 8), square, out=square))
    refused(B.EINVAL, lambda: ops.input_grad(square, f(8, 8), out=square))
    refused(B.EINVAL, lambda: ops.input_grad(f(8, 8), square, out=square))
    refused(B.EINVAL, lambda: ops.weight_grad(square, B.Checkpoint.empty(8, 8), out=square))
    wide = f(8, 16)
    refused(B.EINVAL, lambda: ops.activation_backward(wide[:, :8], dz=wide.view(-1)[:64].view(8, 8)))
    ops.synchronize()
