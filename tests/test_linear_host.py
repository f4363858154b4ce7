"""CPU-only checks of the linear layer: what the library exports, refusals that need no GPU, and the oracle against its own
definition (a gradient is what differences say, a checkpoint is within half a step)."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import oracle.linear_oracle as lo
from paper_2506_17974_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    with open(os.path.join(ROOT, "include", "lqsgd_linear.h")) as fh:
        text = re.sub(r"/\*.*?\*/", "", fh.read(), flags=re.S)
    declared = set(re.findall(r"\b(lqsgd_[a-z_]+)\s*\(", text))
    assert declared == set(B.LINEAR_SYMBOLS), declared ^ set(B.LINEAR_SYMBOLS)
    for name in declared:
        assert hasattr(B.lib(), name), name


def test_header_is_plain_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "lqsgd_linear.h"\nint main(void) { return lqsgd_checkpoint_stride(33) == 64 ? 0 : 1; }\n')
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-fsyntax-only",
                    str(src)], check=True)


@pytest.mark.parametrize("features,stride", [(1, 32), (31, 32), (32, 32), (33, 64), (11008, 11008), (1 << 20, 1 << 20), (0, B.ESHAPE),
                                             (-3, B.ESHAPE), ((1 << 20) + 1, B.ESHAPE)])
def test_checkpoint_stride(features, stride):
    assert B.lib().lqsgd_checkpoint_stride(features) == stride


def test_calls_without_a_context_are_refused():
    L = B.lib()
    assert L.lqsgd_linear_create(None, None) == B.EINVAL
    assert L.lqsgd_linear_synchronize(None) == B.EINVAL
    assert L.lqsgd_linear_destroy(None) == B.OK
    assert L.lqsgd_checkpoint_save(None, 0, 1, 1, None, 1, None, None) == B.EINVAL
    assert L.lqsgd_checkpoint_load(None, 0, 1, 1, None, None, None, 1) == B.EINVAL
    assert L.lqsgd_linear_forward(None, 0, 0, 1, 1, 1, None, 1, None, 1, None, None, 0, None, 1, None, None, None, None) == B.EINVAL
    assert L.lqsgd_linear_activation_backward(None, 0, 0, 1, 1, None, 1, None, None, None, 1, None, 0) == B.EINVAL
    assert L.lqsgd_linear_input_grad(None, 0, 1, 1, 1, None, 1, None, 1, None, 1) == B.EINVAL
    assert L.lqsgd_linear_weight_grad(None, 0, 1, 1, 1, None, 1, None, None, 0, None, 1, 0) == B.EINVAL
    assert L.lqsgd_linear_last_error(None).decode()


def test_no_cpu_path():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is visible")
    with pytest.raises(RuntimeError):
        B.LinearOps()


@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_oracle_checkpoints(kind):
    rng = np.random.default_rng(3)
    v = rng.standard_normal((40, 77)) * np.exp(rng.standard_normal((40, 77)))
    v[0, :] = 0
    v[1, 5] = 127.5 / 64                                  # the boundary itself takes the next exponent
    v[2, 40] = np.inf
    v[3, 70] = np.nan
    if kind == "f16":
        v[4, :] *= 1e-6                                   # below the least exponent: multiples of 2^-24
        v = v.astype(np.float16).astype(np.float64)
    codes, exps = lo.save(v, kind)
    got = lo.load(codes, exps, 77)
    step = np.repeat(np.where(exps == 255, np.nan, 2.0 ** (exps.astype(float) - 127)), 32, 1)[:, :77]
    bad = np.isnan(step)
    assert bad[2, 32:64].all() and bad[3, 64:].all() and bad.sum() == 32 + 13
    assert np.array_equal(np.isnan(got), bad)
    assert (np.abs(got - v)[~bad] <= 0.5 * step[~bad]).all()
    for g in range(3):                                    # no smaller exponent would do
        part = np.abs(v[:, 32 * g:32 * g + 32]).max(1)
        fine = np.isfinite(part) & (exps[:, g] > lo.BOUNDS[kind][0] + 127)
        s = 2.0 ** (exps[fine, g].astype(float) - 127)
        assert (part[fine] < 127.5 * s).all() and (part[fine] >= 127.5 * s / 2).all()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_oracle_gradients_are_the_differences(act):
    """d(sum c y)/dx and /dw along a direction, by central differences of the forward pass at x, w that the gradient is taken at."""
    rng = np.random.default_rng(5)
    x, w, b = rng.standard_normal((6, 9)), rng.standard_normal((7, 9)), rng.standard_normal(7)
    c = rng.standard_normal((6, 7))
    z, _ = lo.forward(x, w, b, act=act)
    dz, db = lo.activation_backward(c, z, act)
    dx, dw = lo.input_grad(dz, w), lo.weight_grad(dz, x)
    ux, uw, ub = rng.standard_normal(x.shape), rng.standard_normal(w.shape), rng.standard_normal(7)
    h = 1e-6
    hi = lo.forward(x + h * ux, w + h * uw, b + h * ub, act=act)[1]
    low = lo.forward(x - h * ux, w - h * uw, b - h * ub, act=act)[1]
    want = float((c * (hi - low)).sum() / (2 * h))
    got = float((dx * ux).sum() + (dw * uw).sum() + (db * ub).sum())
    assert abs(got - want) <= 1e-7 * (1 + abs(want))
