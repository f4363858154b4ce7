"""GPU tests of norms, 8-bit products and dropout of two contexts side by side, and of graphs of them that are replayed on other streams."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear_graphs import Layer

pytestmark = pytest.mark.gpu


class Block(Layer):
    """A context on a stream of its own with calls that use its workspace: an 8-bit product whose sum is in parts, backward passes whose runs are
    joined in the kernel and by another; and dropout by a count on the device."""

    def __init__(self, seed, kind):
        import torch
        self.stream = torch.cuda.Stream()
        with torch.cuda.stream(self.stream):
            self.ops = B.LinearOps()
            g = torch.Generator(device="cuda").manual_seed(seed)
            m, k, n = 64, 11008, 2048
            self.x, self.dy = (torch.randn((m, k), generator=g, device="cuda").to(kind) for _ in range(2))
            self.many = torch.randn((700, 1000), generator=g, device="cuda").to(kind)
            self.small = torch.randn((40, 72), generator=g, device="cuda").to(kind)
            self.w = self.ops.quantize(torch.randn((n, k), generator=g, device="cuda").to(kind))
            self.q, self.count = B.RowCodes.empty(m, k), torch.tensor(seed, device="cuda", dtype=torch.int64)
            self.rstd = [torch.empty(t.shape[0], device="cuda") for t in (self.x, self.many, self.small)]
            empty = torch.empty_like
            self.out = (torch.empty((m, n), dtype=kind, device="cuda"), empty(self.x), empty(self.x), empty(self.many), empty(self.small),
                        torch.empty(k, device="cuda"), torch.empty(1000, device="cuda"), torch.empty(72, device="cuda"))
            self.run()
            self.want = [t.clone() for t in self.out]
            self.stream.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph, stream=self.stream):
                self.run()

    def run(self):
        y, dx, dropped, dx_many, dx_small, *dg = self.out
        self.ops.rms_norm(self.x, rstd=self.rstd[0], quantize_y=self.q, want_y=False)
        self.ops.int8_forward(self.q, self.w, act="gelu", out=y)
        self.ops.dropout(self.x, 0.25, 11, more_offset=self.count, out=dropped)
        self.ops.rms_norm_backward(self.dy, self.x, self.rstd[0], dx=dx, dgain=dg[0])
        for t, rstd, d, g in ((self.many, self.rstd[1], dx_many, dg[1]), (self.small, self.rstd[2], dx_small, dg[2])):
            self.ops.rms_norm(t, rstd=rstd, want_y=False)
            self.ops.rms_norm_backward(t, t, rstd, dx=d, dgain=g)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_replays_on_another_stream_in_order(kind):
    """Replays on a second stream and calls on the context's own, each waiting for what came before."""
    import torch
    print("case: block's graph on another stream", kind, flush=True)
    one, other = Block(3, getattr(torch, kind)), torch.cuda.Stream()
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
    print("case: blocks' contexts side by side", kind, flush=True)
    blocks = [Block(seed, getattr(torch, kind)) for seed in (5, 6, 7)]
    for k in range(6):
        for b in blocks:
            with torch.cuda.stream(b.stream):
                b.clear()
        for _ in range(4):
            for b in blocks:
                with torch.cuda.stream(b.stream):
                    b.graph.replay() if k % 2 else b.run()
        torch.cuda.synchronize()
        assert all(b.right() for b in blocks)
    for b in blocks:
        b.close()
