"""GPU tests of what the linear layer refuses: outputs that start where an input or another output does.  Nothing is launched."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import _say, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
M = N = K = 32


def test_outputs_over_inputs_and_each_other(ops):
    import torch
    _say("overlaps")
    L, h = B.lib(), ops._h
    keep = [torch.zeros(M * K, device="cuda") for _ in range(16)]
    at = [t.data_ptr() for t in keep]
    x, w, bias, r, y, zc, ze, yc, ye, dy, dz, db = at[:12]

    def distinct_or_refused(call, names, outputs, inputs, allowed=()):
        """The call with its own addresses is taken; with an output's put at another's, refused, but for the pairs that may be one."""
        assert call(**names) == B.OK
        for o in outputs:
            for other in inputs + outputs:
                if other != o:
                    want = B.OK if (o, other) in allowed or (other, o) in allowed else B.EINVAL
                    if want == B.OK:
                        continue                        # tested where the results are
                    assert call(**dict(names, **{o: names[other]})) == want, (o, other)
                    assert "output" in L.lqsgd_linear_last_error(h).decode()

    distinct_or_refused(lambda x, codes, exps: L.lqsgd_checkpoint_save(h, 0, M, K, x, K, codes, exps),
                        dict(x=x, codes=zc, exps=ze), ("codes", "exps"), ("x",))
    distinct_or_refused(lambda x, codes, exps: L.lqsgd_checkpoint_load(h, 0, M, K, codes, exps, x, K),
                        dict(x=y, codes=zc, exps=ze), ("x",), ("codes", "exps"))
    distinct_or_refused(lambda x, w, b, r, y, zc, ze, yc, ye: L.lqsgd_linear_forward(h, 0, 2, M, N, K, x, K, w, K, b, r, N, y, N, zc, ze, yc, ye),
                        dict(x=x, w=w, b=bias, r=r, y=y, zc=zc, ze=ze, yc=yc, ye=ye), ("y", "zc", "ze", "yc", "ye"), ("x", "w", "b", "r"),
                        (("y", "r"),))
    distinct_or_refused(lambda dy, zc, ze, dz, db: L.lqsgd_linear_activation_backward(h, 0, 2, M, N, dy, N, zc, ze, dz, N, db, 0),
                        dict(dy=dy, zc=zc, ze=ze, dz=dz, db=db), ("dz", "db"), ("dy", "zc", "ze"), (("dz", "dy"),))
    distinct_or_refused(lambda dz, w, dx: L.lqsgd_linear_input_grad(h, 0, M, N, K, dz, N, w, K, dx, K),
                        dict(dz=dz, w=w, dx=y), ("dx",), ("dz", "w"))
    distinct_or_refused(lambda dz, xc, xe, dw: L.lqsgd_linear_weight_grad(h, 0, M, N, K, dz, N, xc, xe, 0, dw, K, 0),
                        dict(dz=dz, xc=zc, xe=ze, dw=y), ("dw",), ("dz", "xc", "xe"))
    # a checkpoint that an activation does not need is not an input
    assert L.lqsgd_linear_activation_backward(h, 0, 0, M, N, dy, N, zc, ze, zc, N, db, 0) == B.OK
    torch.cuda.synchronize()


def test_checkpoints_over_their_tensors(ops):
    """The same through the binding."""
    import torch
    _say("overlaps of checkpoints")

    def refused(call):
        with pytest.raises(B.LqsgdError) as e:
            call()
        assert e.value.code == B.EINVAL

    raw = torch.zeros(64 * 64 * 4, dtype=torch.uint8, device="cuda")
    x = raw.view(torch.float32).view(64, 64)
    exps = torch.zeros((64, 2), dtype=torch.uint8, device="cuda")
    over = B.Checkpoint(raw[:64 * 64].view(torch.int8).view(64, 64), exps, 64)
    refused(lambda: ops.save(x, out=over))
    refused(lambda: ops.load(over, out=x))
    refused(lambda: ops.forward(x, torch.zeros_like(x), save_z=over))
    z = B.Checkpoint.empty(64, 64)
    refused(lambda: ops.forward(x, torch.zeros_like(x), save_z=z, save_y=z))
    refused(lambda: ops.weight_grad(torch.zeros_like(x), over, out=x))
    refused(lambda: ops.activation_backward(torch.zeros_like(x), over, "relu", dz=x))
