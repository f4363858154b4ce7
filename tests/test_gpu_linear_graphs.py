"""GPU tests of graphs of the linear layer's calls that are replayed on other streams than their context's."""
import pytest

from paper_2506_17974_amd import binding as B

pytestmark = pytest.mark.gpu


class Layer:
    """A context on a stream of its own, forward and backward passes of sizes whose sums are in parts, and a graph of them."""

    def __init__(self, seed, kind):
        import torch
        self.stream = torch.cuda.Stream()
        with torch.cuda.stream(self.stream):
            self.ops = B.LinearOps()
            g = torch.Generator(device="cuda").manual_seed(seed)
            m, n, k = 60, 1000, 3000
            self.x, self.w, self.dz = (torch.randn(s, generator=g, device="cuda").to(kind) for s in ((m, k), (n, k), (m, n)))
            self.held = self.ops.save(self.x)
            self.out = torch.empty((m, n), dtype=kind, device="cuda"), torch.empty((m, k), dtype=kind, device="cuda"), torch.empty((n, k), device="cuda")
            self.run()
            self.want = [t.clone() for t in self.out]
            self.stream.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph, stream=self.stream):
                self.run()

    def run(self):
        y, dx, dw = self.out
        self.ops.forward(self.x, self.w, act="silu", out=y)
        self.ops.input_grad(self.dz, self.w, out=dx)
        self.ops.weight_grad(self.dz, self.held, out=dw)

    def clear(self):
        for t in self.out:
            t.zero_()

    def right(self):
        import torch
        return all(torch.equal(a, b) for a, b in zip(self.want, self.out))

    def close(self):
        del self.graph
        self.ops.close()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_replays_on_another_stream_in_order(kind):
    """Replays on a second stream and calls on the context's own, each waiting for what came before."""
    import torch
    print("case: graph on another stream", kind, flush=True)
    one, other = Layer(3, getattr(torch, kind)), torch.cuda.Stream()
    for _ in range(5):
        other.wait_stream(one.stream)
        with torch.cuda.stream(other):
            one.clear()
            one.graph.replay()
            assert one.right()
        one.stream.wait_stream(other)
        with torch.cuda.stream(one.stream):
            one.clear()
            one.run()
            assert one.right()
    one.close()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_contexts_side_by_side(kind):
    """A context each, graphs and calls on streams that do not wait for each other."""
    import torch
    print("case: contexts side by side", kind, flush=True)
    layers = [Layer(seed, getattr(torch, kind)) for seed in (5, 6, 7)]
    for k in range(6):
        for l in layers:
            with torch.cuda.stream(l.stream):
                l.clear()
        for _ in range(4):
            for l in layers:
                with torch.cuda.stream(l.stream):
                    l.graph.replay() if k % 2 else l.run()
        torch.cuda.synchronize()
        assert all(l.right() for l in layers)
    for l in layers:
        l.close()
