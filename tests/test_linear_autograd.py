"""What autograd makes of the linear layer's calls: a backward() that reaches one raises instead of leaving its gradient out."""
import pytest

from paper_2506_17974_amd import binding as B


def test_marked_results_raise_in_backward():
    """On the CPU: the mark itself."""
    import torch
    x, w = torch.ones(3, 4), torch.ones(2, 4, requires_grad=True)
    out = torch.zeros(3, 2)
    got = B._without_autograd(out, x, w, None)
    assert got is out and out.requires_grad and torch.equal(got, torch.zeros(3, 2))
    got += 1                                            # as any result
    with pytest.raises(B.LqsgdError) as e:
        (got * 2).sum().backward()
    assert e.value.code == B.EINVAL and "weight_grad" in str(e.value)
    for inputs, grad in (((x, w.detach(), None), True), ((x, w), False)):
        out = torch.zeros(3, 2)
        with torch.set_grad_enabled(grad):
            assert B._without_autograd(out, *inputs) is out and not out.requires_grad


@pytest.mark.gpu
def test_calls_on_tensors_that_require_a_gradient():
    import torch
    print("case: autograd", flush=True)
    ops = B.LinearOps()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, b, r = (torch.randn(s, generator=g, device="cuda") for s in ((5, 40), (24, 40), (24,), (5, 24)))
    plain = ops.forward(x, w, b, r, act="gelu")
    assert not plain.requires_grad
    held = ops.save(x)

    def raises(t, want):
        assert torch.equal(t.detach(), want) and t.requires_grad
        with pytest.raises(B.LqsgdError):
            t.sum().backward()

    for k in range(4):
        args = [t.clone().requires_grad_(k == i) for i, t in enumerate((x, w, b, r))]
        raises(ops.forward(*args, act="gelu"), plain)
        with torch.no_grad():
            assert not ops.forward(*args, act="gelu").requires_grad
        out = torch.empty_like(plain)
        assert ops.forward(*args, act="gelu", out=out) is out and not out.requires_grad
    dz, db = ops.activation_backward(r)
    got = ops.activation_backward(r.clone().requires_grad_())
    raises(got[0], dz)
    raises(got[1], db)
    raises(ops.input_grad(r.clone().requires_grad_(), w), ops.input_grad(r, w))
    raises(ops.input_grad(r, w.clone().requires_grad_()), ops.input_grad(r, w))
    raises(ops.weight_grad(r.clone().requires_grad_(), held), ops.weight_grad(r, held))
    # between layers of torch's own, where the weights before the call would have gone without
    first = torch.nn.Linear(40, 40, device="cuda")
    y = ops.forward(first(x), w) @ torch.nn.Linear(24, 3, device="cuda").weight.t()
    with pytest.raises(B.LqsgdError):
        y.sum().backward()
    ops.close()
