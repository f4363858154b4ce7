"""GPU test: the linear layer's calls are refused while another device than the context's is current."""
import pytest

from paper_2506_17974_amd import binding as B

pytestmark = pytest.mark.gpu


def test_calls_while_another_device_is_current():
    """One GPU is enough: what the context asks is made to answer as beside a second one."""
    import torch
    print("case: another device", flush=True)
    ops = B.LinearOps()
    x, w = torch.ones((4, 8), device="cuda"), torch.ones((6, 8), device="cuda")
    dz = torch.ones((4, 6), device="cuda")
    held = ops.save(x)
    calls = [lambda: ops.save(x), lambda: ops.load(held), lambda: ops.forward(x, w), lambda: ops.activation_backward(dz), lambda: ops.input_grad(dz, w),
             lambda: ops.weight_grad(dz, held)]
    if torch.cuda.device_count() > 1:
        with torch.cuda.device((ops.device.index + 1) % torch.cuda.device_count()):
            for call in calls:
                with pytest.raises(B.LqsgdError) as e:
                    call()
                assert e.value.code == B.ESTATE
    asked = ops._current_device
    ops._current_device = lambda: ops.device.index + 1
    for call in calls:
        with pytest.raises(B.LqsgdError) as e:
            call()
        assert e.value.code == B.ESTATE and "device" in str(e.value)
    ops._current_device = lambda: ops.device.index
    for call in calls:
        call()
    ops._current_device = asked
    ops.synchronize()
    ops.close()
