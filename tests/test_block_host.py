"""CPU-only checks of what stands around the linear layer: what the library exports, refusals that need no GPU, and the oracle against
published values, its own definition and differences."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import oracle.block_oracle as bo
from paper_2506_17974_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    with open(os.path.join(ROOT, "include", "lqsgd_block.h")) as fh:
        return fh.read()


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"\b(lqsgd_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", _header(), flags=re.S)))
    assert declared == set(B.BLOCK_SYMBOLS), declared ^ set(B.BLOCK_SYMBOLS)
    for name in declared:
        assert hasattr(B.lib(), name), name


def test_constants():
    assert int(re.search(r"#define LQSGD_INT8_MAX_COLS (\d+)", _header()).group(1)) == B.INT8_MAX_COLS
    assert B.INT8_MAX_COLS * 128 * 128 < 2 ** 31 and B.INT8_MAX_COLS % 32 == 0


def test_header_is_plain_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "lqsgd_block.h"\nint main(void) { return lqsgd_rows_save(0, 0, 1, 1, 0, 1, 0, 0) == LQSGD_EINVAL ? 0 : 1; }\n')
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-fsyntax-only",
                    str(src)], check=True)


def test_calls_without_a_context_are_refused():
    L = B.lib()
    assert L.lqsgd_rows_save(None, 0, 1, 1, None, 1, None, None) == B.EINVAL
    assert L.lqsgd_rows_load(None, 0, 1, 1, None, None, None, 1) == B.EINVAL
    assert L.lqsgd_rms_norm(None, 0, 1, 1, 0.0, None, 1, None, 1, None, None, 1, None, 1, None, None, None, None, None) == B.EINVAL
    assert L.lqsgd_rms_norm_backward(None, 0, 1, 1, None, 1, None, 1, None, None, None, None, None, 1, None, 1, None, 0) == B.EINVAL
    assert L.lqsgd_int8_forward(None, 0, 0, 1, 1, 1, None, None, None, None, None, None, 1, None, 1) == B.EINVAL
    assert L.lqsgd_dropout(None, 0, 1, 1, 0.5, 0, 0, None, None, 1, None, 1, None, 1, None, None) == B.EINVAL
    assert L.lqsgd_linear_last_error(None).decode()


def test_generator_against_published_values():
    """The known answers that its authors publish for Philox 4x32 with 10 rounds: of zeros, of ones, and of digits of pi."""
    ones = 0xFFFFFFFF
    assert bo.philox((0, 0, 0, 0), (0, 0)) == (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)
    assert bo.philox((ones,) * 4, (ones,) * 2) == (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)
    assert bo.philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)


def test_oracle_dropout_keeps_its_share():
    """Of 20000 values with p = 0.3, 14000 stay on average, with a standard deviation of 65: six of them to either side."""
    keep, y = bo.dropout(np.ones((40, 500)), 0.3, 12345, 6)
    assert abs(int(keep.sum()) - 14000) < 390
    assert np.allclose(y[keep], 65536 / (65536 - round(0.3 * 65536)))
    other = bo.dropout(np.ones((40, 500)), 0.3, 12345, 7)[0]
    assert 0.4 < (keep != other).mean() < 0.44               # 2 p (1 - p)
    assert bo.dropout(np.ones((3, 9)), 0.0, 1, 2)[0].all() and not bo.dropout(np.ones((3, 9)), 1.0, 1, 2)[0].any()


def test_oracle_rows():
    rng = np.random.default_rng(3)
    v = (rng.standard_normal((40, 77)) * np.exp(3 * rng.standard_normal((40, 77)))).astype(np.float32)
    v[0, :] = 0
    v[1, 5], v[2, 6] = np.inf, np.nan
    v[3, :] *= np.float32(1e-38)                              # below the least step
    codes, scales = bo.rows_save(v)
    bad = np.isnan(scales)
    assert list(np.flatnonzero(bad)) == [1, 2] and (codes[bad] == 0).all() and (codes[:, 77:] == 0).all() and codes.shape == (40, 96)
    got = bo.rows_load(codes, scales, 77)
    s = scales.astype(np.float64)[:, None]
    assert (np.abs(got - v)[~bad] <= (0.5 + 2.0 ** -16) * np.broadcast_to(s, v.shape)[~bad]).all()
    full = ~bad & (s[:, 0] > 2.0 ** -126)
    assert (np.abs(codes[full]).max(1) == 127).all()


@pytest.mark.parametrize("gain,residual", [(True, True), (False, False)])
def test_oracle_gradients_are_the_differences(gain, residual):
    """d(sum c y + sum d h) along a direction, by central differences of the forward pass."""
    rng = np.random.default_rng(5)
    x, r, c, d = (rng.standard_normal((6, 9)) for _ in range(4))
    g = rng.standard_normal(9) if gain else None
    ux, ug = rng.standard_normal((6, 9)), rng.standard_normal(9)

    def value(t):
        h = x + (r if residual else 0) + t * ux
        return (c * bo.rms_norm(h, None if g is None else g + t * ug, 1e-2)[1]).sum() + (d * h).sum() * residual

    h0 = x + (r if residual else 0)
    rstd, _ = bo.rms_norm(h0, g, 1e-2)
    dx, dg = bo.rms_norm_backward(c, h0, rstd, g, d if residual else None)
    want = (value(1e-5) - value(-1e-5)) / 2e-5
    got = (dx * ux).sum() + ((dg * ug).sum() if gain else 0.0)
    assert abs(got - want) <= 1e-8 * (1 + abs(want))
