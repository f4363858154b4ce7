"""GPU tests of the linear layer with as many samples as it takes."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import _say, _t, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
MOST = 1 << 30


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_the_most_samples(ops, kind):
    """2^30 samples of one feature: more tiles than the kernels of 512 threads can be launched for.  One product a value, rounded once."""
    import torch
    _say("most samples", kind)
    x = torch.randn(MOST, device="cuda", dtype=_t(kind)).view(MOST, 1)
    w = torch.full((1, 1), 1.7, device="cuda", dtype=_t(kind))
    want = x * w
    close = dict(rtol=2.0 ** -21, atol=1e-30) if kind == "f32" else dict(rtol=0, atol=0)      # terms left out: under 2^-22
    got = ops.forward(x, w)
    assert torch.isclose(got, want, **close).all()
    del got
    assert torch.isclose(ops.input_grad(x, w), want, **close).all()


def test_outputs_that_no_launch_holds_are_refused(ops):
    """The sizes are checked before any pointer is used."""
    import torch
    L, h = B.lib(), ops._h
    tensors = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    p, q = (t.data_ptr() for t in tensors)
    wide = 1 << 20
    assert L.lqsgd_linear_forward(h, 0, 0, MOST, wide, 1, p, 1, p, 1, None, None, 0, q, wide, None, None, None, None) == B.ESHAPE
    assert L.lqsgd_linear_input_grad(h, 0, MOST, 1, wide, p, 1, p, wide, q, wide) == B.ESHAPE
    assert L.lqsgd_linear_weight_grad(h, 0, 1, wide, wide, p, wide, p, p, 0, q, wide, 0) == B.ESHAPE
    assert L.lqsgd_linear_last_error(h).decode()
