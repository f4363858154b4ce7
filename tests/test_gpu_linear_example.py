"""examples/train_mlp.py: the operators and the compressor as a training program uses them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_mlp.py")
    spec = importlib.util.spec_from_file_location("train_mlp", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_training_lowers_the_loss(kind):
    import torch
    print("case: train_mlp", kind, flush=True)
    losses = _example().train(torch.float32 if kind == "f32" else torch.bfloat16, steps=30)
    assert abs(losses[0] - 2.5) < 1.0                     # ten classes, nothing learnt yet
    assert losses[-1] < 0.25 * losses[0], losses


def test_gradients_are_autograds():
    """One worker's gradients against torch's own of the same network in float64.  What the 8 bits change: inputs and slopes are off
    by up to half a step, 1/128 to 1/64 of a group's largest value, 0.7 % of a value's size on average and independent, so that the
    gradients, sums over 256 samples, stay within 3 % of their own size."""
    import torch
    from paper_2506_17974_amd import binding as B
    print("case: train_mlp gradients", flush=True)
    ex = _example()
    gen = torch.Generator(device="cuda").manual_seed(7)
    ops = B.LinearOps()
    net = ex.Mlp(ops, gen, torch.float32)
    for b in net.b:
        b.normal_(generator=gen).mul_(0.1)
    x, labels = ex.make_data(1, 256, gen)
    scores, kept = net.forward(x[0])
    loss, g = ex.loss_and_gradient(scores, labels[0])
    dw = [torch.empty(s, device="cuda") for s in ex.LAYERS]
    db = [torch.empty(s[0], device="cuda") for s in ex.LAYERS]
    net.backward(g, kept, dw, db)
    w = [t.double().cpu().requires_grad_() for t in net.w]
    b = [t.double().cpu().requires_grad_() for t in net.b]
    F = torch.nn.functional
    h1 = F.gelu(x[0].double().cpu() @ w[0].t() + b[0])
    h2 = h1 + F.gelu(h1 @ w[1].t() + b[1])
    want = F.cross_entropy(h2 @ w[2].t() + b[2], labels[0].cpu())
    want.backward()
    assert abs(float(loss) - want.item()) < 1e-5
    for got, t in zip(dw + db, w + b):
        assert float((got.double().cpu() - t.grad).norm() / t.grad.norm()) < 0.03
    ops.close()
