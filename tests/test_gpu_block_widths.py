"""GPU tests of rows that end inside a piece of eight values, at every place in it and in every kernel's row: bounds as in test_gpu_block.py."""
import numpy as np
import pytest

import oracle.block_oracle as bo
import tests.test_gpu_block as block
from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import TYPES, _put, _say, ops  # noqa: F401

pytestmark = pytest.mark.gpu

# every end of a piece, and the edges of the kernels' rows: wavefronts' (512, 1024), one piece a thread (4096 to 6144), two with the next row on its
# way (to 12288) and without, four (14336), and rows read twice
WIDTHS = list(range(8, 17)) + [510, 517, 1021, 1028] + list(range(4096, 4105)) + [6143, 6144, 6145, 8191, 8194, 9003, 12287, 12290, 14001, 14341, 32767, 32771]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("features", WIDTHS)
def test_norm(ops, kind, features):
    _say("norm", kind, features)
    block._check_norm(ops, kind, 3, features, 1, 1, residual=True, gain=True)
    block._check_norm(ops, kind, 2, features, 0, 0, residual=False, gain=features % 2 == 0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("features", [f for f in WIDTHS if f < 16000])
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_norm_backward(ops, kind, features, source):
    block.test_norm_backward(ops, kind, 3, features, 1, 1, source)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", [(2000, 4100), (2000, 5000), (1100, 9003), (2600, 65), (9000, 20)])
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_norm_backward_by_even_runs(ops, kind, samples, features, source):
    """More rows than the card's CUs have runs: the runs are made as many for each."""
    block.test_norm_backward(ops, kind, samples, features, 0, 0, source)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("features", list(range(1, 17)) + [125, 510])
def test_rows_and_dropout(ops, kind, features):
    block.test_rows_saved_and_read_back(ops, kind, 3, features, 1, 1)
    block.test_dropout(ops, kind, 3, features, 1, 1, 0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("features", [9, 21, 517, 4101, 9003])
def test_last_values_of_a_row(ops, kind, features):
    """What a row's last piece is read with is not counted twice: large values right before it and in it."""
    _say("last values", kind, features)
    rng = np.random.default_rng(features)
    for at in range(1, 10):
        if at > features:
            continue
        v = rng.standard_normal((2, features))
        v[1, features - at] = 1000.0
        x, hx = _put(v, kind)
        want_r, _ = bo.rms_norm(hx)
        rstd = ops.rms_norm(x, want_rstd=True, want_y=False)[2].cpu().numpy()
        assert (np.abs(rstd - want_r) <= 2 * block.U * want_r).all()
        rows = B.RowCodes.empty(2, features)
        ops.quantize(x, out=rows)
        got, want = block._rows(rows), bo.rows_save(block._fp32(hx))
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
