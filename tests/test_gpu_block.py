"""GPU tests of what stands around the linear layer (include/lqsgd_block.h) against oracle/block_oracle.py.

Tolerances, from the arithmetic (u = 2^-24, half an ulp of fp32):
  rstd              the squares are added up in fp64 and rounded once: u, and another for fp64's own
  y                 two products beside rstd: 4 u of its size, and the rounding to its type
  8-bit rows        codes equal: their definition names every rounding; scales of the norm's rows 3 u
  sums in fp32      u S (8 + 4 sqrt(n)), S = the sum of the magnitudes of n terms
  dx                the sum's error times rstd |h rstd| / n, and 4 roundings of each of its terms
  8-bit products    exact sums; 4 u of what they are multiplied to, u a further addition, and 5e-7 (1 + |z|) for activations
  dropout           the mask equal; 2 u of the product and of the sum
  outputs           rounded once: half an ulp of the type (2^-24, 2^-8, 2^-11 relative; f16 2^-25 absolute below its normal range)
"""
import numpy as np
import pytest

import oracle.block_oracle as bo
import oracle.linear_oracle as lo
from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import TYPES, U, _close, _frame, _held, _host, _put, _rounded, _say, _t, _untouched, ops  # noqa: F401

pytestmark = pytest.mark.gpu

# (samples, features, pad, offset): single values and tokens, edges of pieces, groups, wavefronts and of every kernel's row, long rows
SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (2, 33, 1, 1), (5, 511, 3, 0), (4, 512, 0, 0), (6, 513, 7, 8), (9, 1023, 1, 2), (3, 1025, 0, 3), (7, 2048, 8, 0),
          (1, 2049, 0, 0), (5, 4095, 1, 0), (3, 4096, 0, 0), (2, 4097, 2, 1), (2, 8192, 0, 0), (3, 8200, 8, 0), (2, 16384, 0, 0), (2, 16391, 1, 0),
          (1, 40000, 0, 0), (300, 65, 0, 0), (1100, 24, 0, 0)]


def _values(rng, shape, scale=1.0):
    return rng.standard_normal(shape) * np.exp(rng.standard_normal(shape) * 0.5) * scale


def _vector(a, kind):
    import torch
    v = torch.from_numpy(np.ascontiguousarray(a)).to(_t(kind)).cuda()
    return v, v.double().cpu().numpy()


def _rows(c):
    return c.codes.cpu().numpy(), c.scales.cpu().numpy()


def _from(codes, scales, features):
    import torch
    return B.RowCodes(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), features)


def _fp32(a):
    with np.errstate(over="ignore", under="ignore"):
        return np.asarray(a).astype(np.float32)


# ---------------------------------------------------------------------------
# 8-bit rows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features,pad,offset", SHAPES)
def test_rows_saved_and_read_back(ops, kind, samples, features, pad, offset):
    _say("rows", kind, samples, features, pad, offset)
    rng = np.random.default_rng(features)
    x, hx = _put(_values(rng, (samples, features)), kind, pad, offset)
    q = ops.quantize(x)
    codes, scales = _rows(q)
    want = bo.rows_save(_fp32(hx))
    assert np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])
    for to in TYPES:
        out, flat = _frame((samples, features), to, -7.0, pad, offset)
        assert ops.dequantize(q, out=out) is out
        v = bo.rows_load(codes, scales, features)
        _close(out, v, U * np.abs(v) + _rounded(to, v), "read back")
        assert _untouched(flat, out, -7.0)


@pytest.mark.parametrize("kind", TYPES)
def test_rows_of_special_values(ops, kind):
    import torch
    _say("special rows", kind)
    rng = np.random.default_rng(1)
    v = rng.standard_normal((9, 70))
    v[0] = 0
    v[1, 3], v[2, 69], v[3, 40] = np.inf, np.nan, -np.inf
    v[4] *= 1e-39 if kind == "f32" else 1e-7
    v[5] *= 6e4 if kind == "f16" else 1e38
    v[6] = np.arange(70) - 35.5                                  # ties
    v[7] = -0.0
    v = np.clip(v, -float(torch.finfo(_t(kind)).max), float(torch.finfo(_t(kind)).max), out=v, where=np.isfinite(v))
    x, hx = _put(v, kind)
    got, want = _rows(ops.quantize(x)), bo.rows_save(_fp32(hx))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1], equal_nan=True)
    back = ops.dequantize(ops.quantize(x), _t(kind)).float().cpu().numpy()
    assert np.isnan(back[1:4]).all() and np.isfinite(np.delete(back, (1, 2, 3), 0)).all()


# ---------------------------------------------------------------------------
# the norm
# ---------------------------------------------------------------------------
def _check_norm(ops, kind, samples, features, pad, offset, residual, gain, eps=1e-6, scale=1.0):
    """Every output at once, and each alone the same bits."""
    import torch
    rng = np.random.default_rng(features + samples)
    x, hx = _put(_values(rng, (samples, features), scale), kind, pad, offset)
    r, hr = _put(_values(rng, (samples, features), scale), kind, pad, offset) if residual else (None, 0.0)
    g, hg = _vector(1 + 0.3 * rng.standard_normal(features), kind) if gain else (None, np.ones(features))
    out, flat = _frame((samples, features), kind, -7.0, pad, offset)
    h, flat_h = _frame((samples, features), kind, -7.0, pad, offset) if residual else (None, None)
    held, rows = B.Checkpoint.empty(samples, features), B.RowCodes.empty(samples, features)
    y, got_h, rstd = ops.rms_norm(x, g, r, eps=eps, h=h, out=out, save_y=held, quantize_y=rows, want_rstd=True)
    assert y is out and got_h is h and _untouched(flat, out, -7.0)
    if residual:
        assert _untouched(flat_h, h, -7.0)
        total = hx + hr
        _close(h, total, U * np.abs(total) + _rounded(kind, total), "h")
        hx = h.double().cpu().numpy()
    want_r, want = bo.rms_norm(hx, hg, eps)
    _close(rstd, want_r, 2 * U * want_r, "rstd")
    _close(y, want, 4 * U * np.abs(want) + _rounded(kind, want), "y")
    saved = ops.save(y.contiguous())
    assert torch.equal(saved.codes, held.codes) and torch.equal(saved.exponents, held.exponents)
    codes, scales = _rows(rows)
    wc, ws = bo.rows_save(_fp32(hx) * _fp32(hg))
    assert np.array_equal(codes, wc)
    assert (np.abs(scales - ws * want_r) <= 3 * U * ws * want_r).all()
    alone = ops.rms_norm(x, g, r, eps=eps)
    assert torch.equal(alone[0], y) and alone[2] is None and (not residual or torch.equal(alone[1], h))
    only = B.RowCodes.empty(samples, features)
    none = ops.rms_norm(x, g, r, eps=eps, quantize_y=only, want_y=False, want_h=False)
    assert none == (None, None, None) and torch.equal(only.codes, rows.codes) and torch.equal(only.scales, rows.scales)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features,pad,offset", SHAPES)
def test_norm(ops, kind, samples, features, pad, offset):
    _say("norm", kind, samples, features, pad, offset)
    _check_norm(ops, kind, samples, features, pad, offset, residual=features % 3 != 0, gain=features != 2048)


@pytest.mark.parametrize("kind,scale,eps", [("f32", 1e30, 1e-6), ("f32", 1e-30, 0.0), ("f32", 3e-20, 1e-30), ("bf16", 1e36, 1e-6), ("bf16", 1e-30, 0.0),
                                            ("f16", 100.0, 1e-5), ("f16", 1e-4, 1e-12), ("f32", 1.0, 1e6)])
@pytest.mark.parametrize("features", [70, 5000, 20000])
def test_norm_over_the_range(ops, kind, scale, eps, features):
    _say("norm's range", kind, scale, eps, features)
    _check_norm(ops, kind, 3, features, 0, 0, residual=False, gain=False, eps=eps, scale=scale)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("features", [100, 3000, 17000])
def test_norm_in_place_and_special_rows(ops, kind, features):
    """h over x or over the residual; rows of zeros, with an infinity and with NaN, beside others that they do not touch."""
    import torch
    _say("norm in place", kind, features)
    rng = np.random.default_rng(4)
    v = rng.standard_normal((6, features))
    v[1] = 0
    v[2, 5], v[3, features - 1] = np.inf, np.nan
    x, hx = _put(v, kind)
    r = torch.zeros_like(x)
    want = ops.rms_norm(x, None, r, want_rstd=True)
    for over in (0, 1):
        a, b = x.clone(), r.clone()
        y, h, rstd = ops.rms_norm(a, None, b, h=(a, b)[over], want_rstd=True)
        assert h is (a, b)[over]
        for p, q in zip((y, h, rstd), want):
            assert np.array_equal(p.float().cpu().numpy(), q.float().cpu().numpy(), equal_nan=True)
    y, h, rstd = (t.double().cpu().numpy() for t in want)
    good = [0, 1, 4, 5]
    want_r, want_y = bo.rms_norm(hx[good])
    assert (np.abs(y[good] - want_y) <= 4 * U * np.abs(want_y) + _rounded(kind, want_y)).all()
    assert (y[1] == 0).all() and rstd[2] == 0 and np.isnan(y[2, 5]) and (np.delete(y[2], 5) == 0).all() and np.isnan(y[3]).all() and np.isnan(rstd[3])
    none = ops.rms_norm(x[1:2], eps=0.0)[0]
    assert torch.isnan(none).all()
    rows = B.RowCodes.empty(6, features)
    ops.rms_norm(x, quantize_y=rows, want_y=False)
    codes, scales = _rows(rows)
    assert np.isnan(scales[2:4]).all() and (codes[2:4] == 0).all() and np.isfinite(scales[good]).all() and (codes[1] == 0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features,pad,offset", SHAPES + [(5000, 33, 0, 0), (2100, 520, 0, 0), (1500, 2050, 0, 0)])
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_norm_backward(ops, kind, samples, features, pad, offset, source):
    import torch
    _say("norm backward", kind, samples, features, pad, offset, source)
    rng = np.random.default_rng(features + samples)
    dy, hdy = _put(_values(rng, (samples, features), 0.1), kind, pad, offset)
    x, hx = _put(_values(rng, (samples, features)), kind, pad, offset)
    with_dh, with_gain = features % 2 == 1, features != 2048
    dh, hdh = _put(_values(rng, (samples, features), 0.1), kind, pad, offset) if with_dh else (None, None)
    g, hg = _vector(1 + 0.3 * rng.standard_normal(features), kind) if with_gain else (None, np.ones(features))
    rstd = ops.rms_norm(x, want_rstd=True, want_y=False)[2]
    hr = rstd.double().cpu().numpy()
    if source == "checkpoint":
        x = ops.save(x)
        hx = lo.load(*_host(x), features)
    out, flat = _frame((samples, features), kind, -7.0, pad, offset)
    dx, dg = ops.rms_norm_backward(dy, x, rstd, g, dh=dh, dx=out)
    assert dx is out and _untouched(flat, out, -7.0)
    want, want_g = bo.rms_norm_backward(hdy, hx, hr, hg, hdh)
    v, xh = hdy * hg, hx * hr[:, None]
    along = np.abs(v * xh).mean(1, keepdims=True)
    tol = np.abs(hr[:, None] * xh) * along * U * (8 + 4 * np.sqrt(features))
    tol += 4 * U * (np.abs(hr[:, None]) * (np.abs(v) + np.abs(xh) * along) + (np.abs(hdh) if with_dh else 0))
    _close(dx, want, tol + _rounded(kind, want), "dx")
    tol_g = U * np.abs(hdy * xh).sum(0) * (8 + 4 * np.sqrt(samples)) + U * np.abs(want_g)
    _close(dg, want_g, tol_g, "dgain")
    # each alone, in place, and added to what is there
    again = ops.rms_norm_backward(dy, x, rstd, g, dh=dh, want_dgain=False)
    assert again[1] is None and torch.equal(again[0], dx)
    again = ops.rms_norm_backward(dy, x, rstd, g, dh=dh, want_dx=False)
    assert again[0] is None and torch.equal(again[1], dg)
    more = torch.ones(features, device="cuda")
    ops.rms_norm_backward(dy, x, rstd, g, dh=dh, dx=dy, dgain=more, accumulate=True)
    assert torch.equal(dy, dx)
    _close(more, want_g + 1, tol_g + 2 * U * (1 + np.abs(want_g)), "dgain added")


def test_norm_backward_is_the_differences(ops):
    """fp32: d(sum c y + sum d h) along a direction d of x whose terms add up, by differences of the device's own forward pass: steps of t = 2^-8
    of the values leave a third-order term of about t^2 = 1.5e-5 of the result, and the roundings of y, added up at random, less than that."""
    import torch
    _say("norm's differences")
    rng = np.random.default_rng(8)
    M, N = 40, 600
    x, c, d, g = (torch.from_numpy(rng.standard_normal(s)).float().cuda() for s in ((M, N), (M, N), (M, N), (N,)))
    y, _, rstd = ops.rms_norm(x, g, eps=1e-2, want_rstd=True)
    dx, dg = ops.rms_norm_backward(c, x, rstd, g, dh=d)
    ux, ug, t = dx * (torch.rand_like(dx) + 0.5), dg / dg.norm() * g.norm() / 8, 2.0 ** -8
    ux = ux / ux.norm() * x.norm()

    def value(s):
        xs = x + s * ux
        return float((c.double() * ops.rms_norm(xs, g + s * ug, eps=1e-2)[0].double()).sum() + (d.double() * xs.double()).sum())

    want = (value(t) - value(-t)) / (2 * t)
    got = float((dx.double() * ux.double()).sum() + (dg.double() * ug.double()).sum())
    assert abs(got - want) <= 2e-4 * abs(want), (got, want)


# ---------------------------------------------------------------------------
# the linear layer on 8-bit rows
# ---------------------------------------------------------------------------
INT8 = [(1, 1, 1), (1, 10, 512), (1, 257, 1155), (2, 64, 27), (3, 5, 7), (4, 1000, 2049), (5, 33, 65), (7, 129, 131), (13, 64, 800), (16, 96, 256), (17, 32, 25),
        (31, 31, 33), (33, 65, 33), (64, 1024, 96), (65, 10, 1024), (127, 128, 127), (129, 127, 64), (255, 256, 257), (256, 257, 255), (300, 257, 513),
        (511, 40, 8), (640, 384, 320), (1000, 16, 16), (33, 200, 4096), (96, 4096, 40), (9000, 10, 33), (5, 10, 11008), (40, 500, 11008), (520, 520, 2080)]


def _check_int8(ops, kind, M, N, K, act, bias, residual, codes=None):
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    if codes is None:
        xc, xs = bo.rows_save(_fp32(_values(rng, (M, K))))
        wc, ws = bo.rows_save(_fp32(_values(rng, (N, K), K ** -0.5)))
    else:
        xc, xs, wc, ws = codes
    b, hb = _vector(0.3 * rng.standard_normal(N), kind) if bias else (None, np.zeros(N))
    r, hr = _put(rng.standard_normal((M, N)), kind, 3, 1) if residual else (None, np.zeros((M, N)))
    out, flat = _frame((M, N), kind, -7.0, 5, 1)
    got = ops.int8_forward(_from(xc, xs, K), _from(wc, ws, K), b, r, act=act, out=out)
    assert got is out and _untouched(flat, out, -7.0)
    p = bo.int8_sums(xc, wc) * (xs.astype(np.float64)[:, None] * ws.astype(np.float64))
    z = p + hb
    y = lo.activate(z, act) + hr
    tol = 4 * U * np.abs(p) + U * np.abs(z)
    tol = 1.2 * tol + (5e-7 * (1 + np.abs(z)) if act != "none" else 0)          # 1.2: the largest slope of an activation, 1.13
    _close(out, y, tol + U * np.abs(y) + _rounded(kind, y), "y")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,N,K", INT8)
def test_int8_forward(ops, kind, M, N, K):
    act = ("none", "relu", "gelu", "silu")[(M + N + K) % 4]
    _say("int8", kind, M, N, K, act)
    _check_int8(ops, kind, M, N, K, act, bias=N % 2 == 0, residual=K % 2 == 1)


@pytest.mark.parametrize("M,N", [(1, 40), (20, 33), (70, 70), (300, 130)])
@pytest.mark.parametrize("K", [16384, 131040])
def test_int8_largest_sums(ops, M, N, K):
    """Every code at its largest, -128 among them: the sums need 32 bits."""
    _say("int8 largest", M, N, K)
    if M * N * K > 1 << 29:
        M = 70
    xc, wc = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
    wc[1::2] = 127
    one = (np.ones(M, np.float32), np.full(N, 2.0 ** -20, np.float32))
    _check_int8(ops, "f32", M, N, K, "none", False, False, (xc, one[0], wc, one[1]))


def test_int8_special_scales(ops):
    """A NaN scale reaches its sample's or its feature's outputs and no others; the sums over no samples are none."""
    import torch
    _say("int8 special")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn((40, 300), generator=g, device="cuda"), torch.randn((70, 300), generator=g, device="cuda")
    clean = ops.int8_forward(ops.quantize(x), ops.quantize(w), act="silu", dtype=torch.float32)
    x[3, 7], w[11, 0] = float("nan"), float("inf")
    y = ops.int8_forward(ops.quantize(x), ops.quantize(w), act="silu", dtype=torch.float32)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[3], bad[:, 11] = True, True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])
    assert ops.int8_forward(ops.quantize(x[:0]), ops.quantize(w)).shape == (0, 70)
    r = clean.clone()
    assert torch.equal(ops.int8_forward(ops.quantize(x[:3]), ops.quantize(w[:11]), residual=r[:3, :11], out=r[:3, :11]),
                       ops.int8_forward(ops.quantize(x[:3]), ops.quantize(w[:11]), residual=clean[:3, :11]))


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features,pad,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (2, 33, 1, 1), (5, 511, 3, 0), (6, 64, 7, 8), (40, 24, 0, 3), (17, 300, 0, 0)])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_dropout(ops, kind, samples, features, pad, offset, p):
    import torch
    _say("dropout", kind, samples, features, pad, offset, p)
    rng = np.random.default_rng(features)
    x, hx = _put(_values(rng, (samples, features)), kind, pad, offset)
    r, hr = _put(_values(rng, (samples, features)), kind, pad, offset) if features % 2 else (None, None)
    seed, off = (1 << 63) + 12345 * features, (3 << 32) + 17
    out, flat = _frame((samples, features), kind, -7.0, pad, offset)
    held = B.Checkpoint.empty(samples, features)
    assert ops.dropout(x, p, seed, off, residual=r, out=out, save_y=held) is out
    keep, want = bo.dropout(hx, p, seed, off, hr)
    _close(out, want, 2 * U * (np.abs(want) + np.abs(hr if hr is not None else 0)) + U * np.abs(want) + _rounded(kind, want), "y")
    assert _untouched(flat, out, -7.0)
    if r is None:
        assert np.array_equal(out.float().cpu().numpy() != 0, keep & (hx != 0))
    saved = ops.save(out.contiguous())
    assert torch.equal(saved.codes, held.codes) and torch.equal(saved.exponents, held.exponents)
    # without the checkpoint, onto the residual or in place; the offset from the device
    more = torch.tensor(5, device="cuda", dtype=torch.int64)
    assert torch.equal(ops.dropout(x, p, seed, off - 5, residual=r, more_offset=more), out)
    over = (r if r is not None else x).clone()
    assert torch.equal(ops.dropout(x if r is not None else over, p, seed, off, residual=over if r is not None else None, out=over), out)


def test_dropout_ends_and_special_values(ops):
    import torch
    _say("dropout's ends")
    x = torch.full((9, 40), float("nan"), device="cuda")
    x[::2] = float("inf")
    r = torch.randn_like(x)
    assert torch.equal(ops.dropout(x, 1.0, 3, residual=r), r) and (ops.dropout(x, 1.0, 3) == 0).all()
    assert torch.equal(ops.dropout(r, 0.0, 3), r)
    keep, _ = bo.dropout(np.ones((9, 40)), 0.4, 3, 0)
    got = ops.dropout(x, 0.4, 3).cpu().numpy()
    assert np.array_equal(got == 0, ~keep) and np.isnan(got[1::2][keep[1::2]]).all() and np.isinf(got[::2][keep[::2]]).all()
    # 64 bits of seed and offset count, and wrap where the device adds
    keeps = [ops.dropout(torch.ones(4, 512, device="cuda"), 0.5, s, o) for s, o in ((1, 0), (1 << 32, 0), (1, 1 << 32), (1, 1), (2, 0))]
    assert all(not torch.equal(a, b) for i, a in enumerate(keeps) for b in keeps[:i])
    more = torch.tensor(1, device="cuda", dtype=torch.int64)
    ones = torch.ones(4, 512, device="cuda")
    assert torch.equal(ops.dropout(ones, 0.5, 1, (1 << 64) - 1, more_offset=more), keeps[0])


@pytest.mark.parametrize("kind", TYPES)
def test_dropout_share_and_gradient(ops, kind):
    """The gradient of x is the same call on dy: y is linear in x, so <dy, y> = <dx, x> up to roundings; and the share that stays (six standard
    deviations)."""
    import torch
    _say("dropout's share", kind)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn((700, 1000), generator=g, device="cuda").to(_t(kind)) for _ in range(2))
    for p in (0.05, 0.25, 0.9):
        y, dx = ops.dropout(x, p, 99, 4), ops.dropout(dy, p, 99, 4)
        kept, n = int((y != 0).sum() + (x == 0).sum()), x.numel()
        assert abs(kept - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5 + n * 2.0 ** -17 + int((x == 0).sum())
        a, b = (dy.double() * y.double()), (dx.double() * x.double())
        tol = _rounded(kind, 1.0)[()] * (a.abs().sum() + b.abs().sum()) + 2.0 ** -24 * dy.abs().double().sum()
        assert abs(float(a.sum() - b.sum())) <= float(tol)


# ---------------------------------------------------------------------------
# large tensors, which are read past the caches
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind,samples,features", [("bf16", 8200, 4099), ("f16", 70000, 481), ("f32", 4100, 4101), ("bf16", 3300, 11003), ("f32", 2050, 9001)])
def test_large_tensors_row_by_row(ops, kind, samples, features):
    """Norm, rows, the norm's backward and dropout of 64 MiB and more against the same calls on parts of the rows, bit by bit; dgain, whose sum
    is over all of them, against float64."""
    import torch
    _say("large", kind, samples, features)
    g = torch.Generator(device="cuda").manual_seed(samples)
    x, r, dy, dh = (torch.randn((samples, features), generator=g, device="cuda").to(_t(kind)) for _ in range(4))
    assert x.numel() * x.element_size() >= 1 << 26
    gain = (torch.randn(features, generator=g, device="cuda") * 0.2 + 1).to(_t(kind))
    held, rows = B.Checkpoint.empty(samples, features), B.RowCodes.empty(samples, features)
    y, h, rstd = ops.rms_norm(x, gain, r, save_y=held, quantize_y=rows, want_rstd=True)
    q = ops.quantize(x)
    dx, dg = ops.rms_norm_backward(dy, h, rstd, gain, dh=dh)
    drop = ops.dropout(x, 0.2, 77, 5, residual=r)
    for part in (slice(0, 9), slice(samples // 2, samples // 2 + 130), slice(samples - 7, samples)):
        c, b = B.Checkpoint.empty(x[part].shape[0], features), B.RowCodes.empty(x[part].shape[0], features)
        want = ops.rms_norm(x[part], gain, r[part], save_y=c, quantize_y=b, want_rstd=True)
        for got, w in zip((y, h, rstd, held.codes, held.exponents, rows.codes, rows.scales), want + (c.codes, c.exponents, b.codes, b.scales)):
            assert torch.equal(got[part], w)
        w = ops.quantize(x[part])
        assert torch.equal(q.codes[part], w.codes) and torch.equal(q.scales[part], w.scales)
        assert torch.equal(dx[part], ops.rms_norm_backward(dy[part], h[part], rstd[part], gain, dh=dh[part], want_dgain=False)[0])
    assert torch.equal(drop[:50], ops.dropout(x[:50], 0.2, 77, 5, residual=r[:50]))
    hx, hr = x[:3].double().cpu().numpy(), r[:3].double().cpu().numpy()
    keep, want = bo.dropout(hx, 0.2, 77, 5, hr)
    _close(drop[:3], want, 2 * U * (np.abs(want) + np.abs(hr)) + U * np.abs(want) + _rounded(kind, want), "dropout")
    assert np.array_equal(drop[:3].double().cpu().numpy()[~keep], hr[~keep])
    terms = dy.double() * h.double() * rstd.double()[:, None]
    want, size = terms.sum(0), terms.abs().sum(0)
    assert ((dg.double() - want).abs() <= U * size * (8 + 4 * samples ** 0.5)).all()


@pytest.mark.parametrize("kind,source", [("f16", "tensor"), ("bf16", "checkpoint"), ("f32", "tensor")])
def test_more_samples_than_a_launch_takes(ops, kind, source):
    """2^21 rows and some: norm, rows and the norm's backward go in parts, whose sums add up."""
    import torch
    _say("many samples", kind, source)
    samples, features = (1 << 21) + 777, 9
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn((samples, features), generator=g, device="cuda").to(_t(kind)) for _ in range(2))
    y, _, rstd = ops.rms_norm(x, want_rstd=True)
    q = ops.quantize(x)
    h = ops.save(x) if source == "checkpoint" else x
    before = torch.randn(features, generator=g, device="cuda")
    dg = before.clone()
    dx, _ = ops.rms_norm_backward(dy, h, rstd, dgain=dg, accumulate=True)
    for part in (slice(0, 40), slice((1 << 21) - 20, (1 << 21) + 20), slice(samples - 40, samples)):
        w = ops.rms_norm(x[part], want_rstd=True)
        assert torch.equal(y[part], w[0]) and torch.equal(rstd[part], w[2])
        c = ops.quantize(x[part])
        assert torch.equal(q.codes[part], c.codes) and torch.equal(q.scales[part], c.scales)
        hp = ops.save(x[part]) if source == "checkpoint" else x[part]
        assert torch.equal(dx[part], ops.rms_norm_backward(dy[part], hp, rstd[part], want_dgain=False)[0])
    held = ops.load(h, torch.float32) if source == "checkpoint" else x
    terms = dy.double() * held.double() * rstd.double()[:, None]
    want, size = terms.sum(0) + before.double(), terms.abs().sum(0)
    assert ((dg.double() - want).abs() <= U * size * (8 + 4 * samples ** 0.5) + U * want.abs()).all()


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
def test_block_as_it_is_used(ops, kind):
    """A block's forward and backward pass with the linear layer's calls: norm, widening layer with gelu, narrowing layer, dropout onto the
    residual stream; checkpoints feed the weight gradients.  Each gradient against the formulas at what the device's tensors hold."""
    import torch
    _say("block", kind)
    T = _t(kind)
    gen = torch.Generator(device="cuda").manual_seed(6)
    M, D, F = 48, 96, 200

    def new(*s, scale=1.0):
        return (torch.randn(s, generator=gen, device="cuda") * scale).to(T)

    x, gain, w1, b1, w2 = new(M, D), 1 + new(D, scale=0.1), new(F, D, scale=D ** -0.5), new(F, scale=0.1), new(D, F, scale=F ** -0.5)
    k1, z1, k2 = B.Checkpoint.empty(M, D), B.Checkpoint.empty(M, F), B.Checkpoint.empty(M, F)
    y, _, rstd = ops.rms_norm(x, gain, save_y=k1, want_rstd=True)
    a = ops.forward(y, w1, b1, act="gelu", save_z=z1, save_y=k2)
    o = ops.forward(a, w2)
    out = ops.dropout(o, 0.25, 11, 3, residual=x)
    want = bo.dropout(o.double().cpu().numpy(), 0.25, 11, 3, x.double().cpu().numpy())[1]
    _close(out, want, 4 * U * (np.abs(want) + 3) + _rounded(kind, want), "out")
    dout = new(M, D, scale=0.1)
    do = ops.dropout(dout, 0.25, 11, 3)
    dw2 = ops.weight_grad(do, k2)
    da = ops.input_grad(do, w2)
    dz, db1 = ops.activation_backward(da, z1, "gelu")
    dw1 = ops.weight_grad(dz, k1)
    dy = ops.input_grad(dz, w1)
    dx, dg = ops.rms_norm_backward(dy, x, rstd, gain, dh=dout)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    wdx, wdg = bo.rms_norm_backward(f(dy), f(x), f(rstd), f(gain), f(dout))
    assert (np.abs(f(dx) - wdx) <= 1e-5 * (1 + np.abs(wdx)) + _rounded(kind, wdx)).all()
    assert (np.abs(f(dg) - wdg) <= U * (8 + 4 * M ** 0.5) * np.abs(f(dy) * f(x) * f(rstd)[:, None]).sum(0) + U * np.abs(wdg)).all()
    wdw = lo.weight_grad(f(dz), lo.load(*_host(k1), D))
    assert (np.abs(f(dw1) - wdw) <= U * (8 + 4 * M ** 0.5) * (np.abs(f(dz)).T @ np.abs(lo.load(*_host(k1), D))) + U * np.abs(wdw)).all()
    # the same layer served from 8-bit rows: what the codes stand for, multiplied in float64
    rows, q1 = B.RowCodes.empty(M, D), ops.quantize(w1)
    ops.rms_norm(x, gain, quantize_y=rows, want_y=False)
    served = ops.int8_forward(rows, q1, b1, act="gelu", dtype=T)
    z = bo.rows_load(*_rows(rows), D) @ bo.rows_load(*_rows(q1), D).T + f(b1)
    want = lo.activate(z, "gelu")
    assert (np.abs(f(served) - want) <= 1e-6 * (1 + np.abs(z)) + _rounded(kind, want)).all()
    for t in (dw2, db1):
        assert torch.isfinite(t).all()


# ---------------------------------------------------------------------------
# graphs
# ---------------------------------------------------------------------------
def test_graph_of_a_block(ops):
    """Norm, 8-bit product, dropout with an offset that the graph counts up, norm's backward: every replay against the same calls made
    one by one, with other work between."""
    import torch
    _say("graph of a block")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        mine = B.LinearOps()
        g = torch.Generator(device="cuda").manual_seed(9)
        x, r, dy = (torch.randn((50, 1000), generator=g, device="cuda") for _ in range(3))
        w = mine.quantize(torch.randn((1000, 1000), generator=g, device="cuda"))
        count = torch.zeros((), dtype=torch.int64, device="cuda")
        rows, rstd, dg = B.RowCodes.empty(50, 1000), torch.empty(50, device="cuda"), torch.empty(1000, device="cuda")
        outs = [torch.empty_like(x) for _ in range(4)]

        def run():
            count.add_(1)
            mine.rms_norm(x, None, r, h=outs[0], rstd=rstd, quantize_y=rows, want_y=False)
            mine.int8_forward(rows, w, out=outs[1])
            mine.dropout(outs[1], 0.5, 7, more_offset=count, out=outs[2])
            mine.rms_norm_backward(dy, outs[0], rstd, dx=outs[3], dgain=dg)

        run()
        stream.synchronize()
        count.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        masks = []
        for k in range(1, 5):
            x.normal_(generator=g)
            count.fill_(k - 1)
            run()
            want = [t.clone() for t in outs + [dg, rstd, rows.codes, rows.scales]]
            for t in outs:
                t.zero_()
            count.fill_(k - 1)
            stream.synchronize()
            graph.replay()
            got = outs + [dg, rstd, rows.codes, rows.scales]
            assert all(torch.equal(a, b) for a, b in zip(got, want)) and int(count) == k
            masks.append((outs[2] != 0).clone())
        assert all(not torch.equal(a, b) for i, a in enumerate(masks) for b in masks[:i])
        stream.synchronize()
        del graph
        mine.close()
