"""GPU tests of the norm at the ends of the types' range, where 1 / sqrt(mean h^2 + eps) or h gain are not normal fp32 numbers but y is.

Tolerances: those of tests/test_gpu_block.py, and beside them half of the least step (2^-149 times the gain for a product below the normal range, the
type's own for the output)."""
import numpy as np
import pytest

import oracle.block_oracle as bo
from paper_2506_17974_amd import binding as B
from tests.test_gpu_block import U, _fp32, _rows, _vector
from tests.test_gpu_linear import _put, _rounded, _say, _t, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133}


def _check(ops, kind, h, gain, eps, x=None, residual=None):
    """y, its checkpoint and its 8-bit rows, of a tensor (or of a sum, h over x) whose values h holds."""
    import torch
    samples, features = h.shape
    x, hx = _put(h, kind) if x is None else (x, h)
    g, hg = (None, np.ones(features)) if gain is None else _vector(gain, kind)
    held, rows = B.Checkpoint.empty(samples, features), B.RowCodes.empty(samples, features)
    y, _, rstd = ops.rms_norm(x, g, residual, eps=eps, h=None if residual is None else x, save_y=held, quantize_y=rows, want_rstd=True)
    want_r, want = bo.rms_norm(hx, hg, eps)
    got = y.double().cpu().numpy()
    tol = 4 * U * np.abs(want) + _rounded(kind, want) + LEAST["f32"] * (1 + np.abs(hg)) + LEAST[kind]
    assert np.isfinite(want).all() and (np.abs(got - want) <= tol).all()
    saved = ops.save(y)
    assert torch.equal(saved.codes, held.codes) and torch.equal(saved.exponents, held.exponents)
    fits = want_r < 2.0 ** 128
    r = rstd.double().cpu().numpy()
    assert (np.abs(r - want_r)[fits] <= 2 * U * want_r[fits] + LEAST["f32"]).all() and np.isinf(r[~fits]).all()
    codes, scales = _rows(rows)
    wc, ws = bo.norm_rows(hx, hg, eps)
    assert np.array_equal(codes, wc)
    assert (np.abs(scales - ws) <= 3 * U * ws + LEAST["f32"]).all() and np.isfinite(scales).all()
    back = bo.rows_load(codes, scales, features)
    full = np.abs(want).max(1) > 2.0 ** -118                                   # rows whose step is not the least one
    assert (np.abs(codes[full]).max(1) == 127).all()
    assert (np.abs(back - want) <= (0.5 + 2.0 ** -16) * ws[:, None] + 4 * U * np.abs(want)).all()
    only = B.RowCodes.empty(samples, features)
    if residual is None:
        ops.rms_norm(x, g, eps=eps, quantize_y=only, want_y=False)
        assert torch.equal(only.codes, rows.codes) and torch.equal(only.scales, rows.scales)
        assert torch.equal(ops.rms_norm(x, g, eps=eps)[0], y)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("features", [7, 70, 600, 5000, 9000, 33000])
@pytest.mark.parametrize("scale", [1e-37, 2e-38, 1.2e-38, 4e-39, 2e-39, 3e-40, 2e-44, 3e37, 8e37, 1e38])
def test_norm_of_rows_as_small_and_as_large_as_there_are(ops, kind, scale, features):
    _say("norm's ends", kind, scale, features)
    rng = np.random.default_rng(features)
    h = np.clip(rng.standard_normal((3, features)), -3, 3) * scale
    h[:, 0] = scale                                                            # no row of zeros alone, whatever the type keeps
    if kind == "bf16":
        h[:, 0] = max(scale, 2.0 ** -133)
    gain = 1 + 0.3 * rng.standard_normal(features)
    for g in (None, gain):
        _check(ops, kind, h, g, 0.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("features", [70, 5000, 33000])
@pytest.mark.parametrize("size,gain,eps", [(1e-37, 1.0, 1e-6), (1e-20, 1e-19, 1e-30), (1e20, 1e25, 1e-6), (1e10, 3e36, 0.0), (1.0, 1e-36, 1e-6), (1.0, 1e-37, 0.0), (1e-30, 1e-3, 1e-80)])
def test_rows_whose_products_with_the_gain_leave_the_range(ops, kind, size, gain, eps, features):
    """h gain below what the least step resolves or beyond fp32, while y is neither; and gains that make y itself small."""
    _say("norm's products", kind, size, gain, eps, features)
    rng = np.random.default_rng(features + 1)
    h = np.clip(rng.standard_normal((3, features)), -3, 3) * size
    h[1] *= 1e-3
    _check(ops, kind, h, np.clip(1 + 0.3 * rng.standard_normal(features), 0.1, 2) * gain, eps)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("features", [70, 5000, 33000])
def test_rows_of_zeros_with_the_least_eps(ops, kind, features):
    """0 times a finite root is 0, however small eps is; with eps = 0 it is NaN, as the formula has it."""
    import torch
    _say("zeros and eps", kind, features)
    x = torch.zeros((3, features), device="cuda", dtype=_t(kind))
    x[1, 3] = 1.0
    for eps in (1e-76, 1e-80, 1e-200, 5e-324):
        rows = B.RowCodes.empty(3, features)
        y = ops.rms_norm(x, eps=eps, quantize_y=rows)[0]
        assert not y[0].any() and not y[2].any() and not rows.codes[::2].any() and torch.isfinite(rows.scales).all()
        assert abs(float(y[1, 3]) - features ** 0.5) <= features ** 0.5 * _rounded(kind, 1.0)[()] * 1.1
    rows = B.RowCodes.empty(3, features)
    y = ops.rms_norm(x, eps=0.0, quantize_y=rows)[0]
    assert torch.isnan(y[::2]).all() and torch.isfinite(y[1]).all()


@pytest.mark.parametrize("features", [70, 5000, 33000])
@pytest.mark.parametrize("scale", [3e-40, 1e38])
def test_sum_over_its_input(ops, features, scale):
    """h over x, rows read again for the widest: what is scaled is the sum."""
    import torch
    _say("norm's ends, in place", features, scale)
    rng = np.random.default_rng(features + 2)
    a, b = (np.clip(rng.standard_normal((2, features)), -1.2, 1.2) * scale for _ in range(2))
    x, r = (torch.from_numpy(_fp32(v)).cuda() for v in (a, b))
    h = (x + r).double().cpu().numpy()
    _check(ops, "f32", h, 1 + 0.1 * rng.standard_normal(features), 0.0, x, r)
