"""GPU tests of what autograd makes of the calls around the linear layer: a backward() that reaches one raises, whatever required the gradient, and
forward-mode tangents are refused rather than left out."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import _say, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu


def _needs(t):
    return t.clone().requires_grad_()


def _raises_in_backward(t):
    assert t.requires_grad
    with pytest.raises(B.LqsgdError) as e:
        t.sum().backward()
    assert e.value.code == B.EINVAL


def test_empty_batch_from_a_checkpoint(ops):
    """No samples, h from a checkpoint: the gradients of sums over nothing are zeros, and marked like those of any batch."""
    import torch
    _say("autograd, empty batch")
    dy, rstd, gain = torch.empty((0, 40), device="cuda"), torch.empty(0, device="cuda"), torch.randn(40, device="cuda")
    held = B.Checkpoint.empty(0, 40)
    dx, dgain = ops.rms_norm_backward(dy, held, rstd, gain)
    assert dx.shape == (0, 40) and not dgain.any() and not dgain.requires_grad
    for args in ((_needs(dy), rstd, gain), (dy, _needs(rstd), gain), (dy, rstd, _needs(gain))):
        dx, dgain = ops.rms_norm_backward(args[0], held, *args[1:])
        assert dx.shape == (0, 40) and not dgain.any()
        _raises_in_backward(dx)
        _raises_in_backward(dgain)


def test_empty_residual(ops):
    """No samples: a residual of none is an input as any other."""
    import torch
    _say("autograd, empty residual")
    x, w = torch.empty((0, 40), device="cuda"), torch.randn((40, 40), device="cuda")
    r, q = _needs(x), ops.quantize(w)
    for out in (*ops.rms_norm(x, residual=r)[:2], ops.forward(x, w, residual=r), ops.int8_forward(ops.quantize(x), q, residual=r), ops.dropout(x, 0.5, 1, residual=r)):
        assert out.shape == (0, 40)
        _raises_in_backward(out)


def test_scales_that_require_a_gradient(ops):
    """Scales of 8-bit rows given as tensors are inputs like the others."""
    import torch
    _say("autograd, scales")
    q, w = (ops.quantize(torch.randn((5, 40), device="cuda")) for _ in range(2))
    plain = ops.int8_forward(q, w, dtype=torch.float32)
    mine = [B.RowCodes(c.codes, _needs(c.scales), 40) for c in (q, w)]
    assert not plain.requires_grad and not ops.dequantize(q).requires_grad
    for args in ((mine[0], w), (q, mine[1])):
        y = ops.int8_forward(*args, dtype=torch.float32)
        assert torch.equal(y.detach(), plain)
        _raises_in_backward(y)
    _raises_in_backward(ops.dequantize(mine[0]))
    q.scales.requires_grad_()                                 # of one made by the calls, too
    _raises_in_backward(ops.dequantize(q))
    with torch.no_grad():
        assert not ops.dequantize(q).requires_grad and not ops.int8_forward(q, mine[1]).requires_grad
    out = torch.empty((5, 40), device="cuda")
    assert ops.dequantize(mine[0], out=out) is out and not out.requires_grad       # plain memory


def test_forward_mode_tangents(ops):
    """A tangent on an input of what would be a new tensor is refused; tensors given for the results are plain memory, here too."""
    import torch
    import torch.autograd.forward_ad as ad
    _say("autograd, tangents")
    g = torch.Generator(device="cuda").manual_seed(4)
    x, r, w = (torch.randn((40, 40), generator=g, device="cuda") for _ in range(3))
    gain = torch.randn(40, generator=g, device="cuda")
    held, q = ops.save(x), ops.quantize(x)
    rstd = ops.rms_norm(x, want_rstd=True, want_y=False)[2]
    calls = {                                                # what is called, and its inputs
        "forward": (lambda a, b, c, d: ops.forward(a, b, c, d), (x, w, gain, r)),
        "activation_backward": (lambda a: ops.activation_backward(a), (x,)),
        "input_grad": (lambda a, b: ops.input_grad(a, b), (x, w)),
        "weight_grad": (lambda a: ops.weight_grad(a, held), (x,)),
        "rms_norm": (lambda a, b, c: ops.rms_norm(a, b, c), (x, gain, r)),
        "rstd alone": (lambda a: ops.rms_norm(a, want_y=False, want_rstd=True), (x,)),
        "h alone": (lambda a, b: ops.rms_norm(a, residual=b, out=torch.empty_like(x)), (x, r)),
        "rms_norm_backward": (lambda a, b, c, d, e: ops.rms_norm_backward(a, b, c, d, e), (x, w, rstd, gain, r)),
        "dgain alone": (lambda a, b, c: ops.rms_norm_backward(a, held, b, c, want_dx=False), (x, rstd, gain)),
        "dequantize": (lambda s: ops.dequantize(B.RowCodes(q.codes, s, 40)), (q.scales,)),
        "int8_forward": (lambda a, b, c, d: ops.int8_forward(B.RowCodes(q.codes, c, 40), B.RowCodes(q.codes, d, 40), a, b), (gain, r, q.scales, q.scales)),
        "dropout": (lambda a, b: ops.dropout(a, 0.5, 1, residual=b), (x, r)),
    }
    for name, (call, args) in calls.items():
        call(*args)
        with ad.dual_level():
            call(*args)                                      # a level without tangents is no matter
            for k in range(len(args)):
                duals = [ad.make_dual(t, torch.ones_like(t)) if i == k else t for i, t in enumerate(args)]
                with pytest.raises(B.LqsgdError) as e:
                    call(*duals)
                assert e.value.code == B.EINVAL and "tangent" in str(e.value), (name, k)
    with ad.dual_level():
        d, out = ad.make_dual(x, torch.ones_like(x)), torch.empty_like(x)
        assert ops.rms_norm(d, out=out)[0] is out and ad.unpack_dual(out).tangent is None
        ops.save(d, out=held)
        ops.quantize(d, out=q)
        ops.rms_norm(d, quantize_y=q, want_y=False)
    with pytest.raises(Exception):                           # a transform's own tensors have no memory
        torch.func.jvp(lambda t: ops.rms_norm(t)[0], (x,), (x,))
