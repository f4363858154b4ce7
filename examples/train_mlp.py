"""Data-parallel training of a small residual network on one GPU: every worker's layers run on the linear-layer operators, keep
their inputs and pre-activations in 8 bits, and write their gradients straight into the buffers that the LQ-SGD compressor reads;
one step_update exchanges the compressed gradients and updates the parameters.

    python examples/train_mlp.py [--type f32|bf16] [--steps N]

    h1 = gelu(x W1^T + b1);  h2 = h1 + gelu(h1 W2^T + b2);  scores = h2 W3^T + b3;  loss = cross entropy, mean over the samples
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

from paper_2506_17974_amd import binding as B

FEATURES, HIDDEN, CLASSES = 784, 512, 10
LAYERS = [(HIDDEN, FEATURES), (HIDDEN, HIDDEN), (CLASSES, HIDDEN)]      # rows x cols: output x input features
ACTS = ["gelu", "gelu", "none"]


def make_data(workers, samples, gen):
    """Classes as noisy clusters, the same for every worker."""
    centres = torch.randn((CLASSES, FEATURES), generator=gen, device="cuda")
    labels = torch.randint(0, CLASSES, (workers, samples), generator=gen, device="cuda")
    return centres[labels] * 0.2 + torch.randn((workers, samples, FEATURES), generator=gen, device="cuda"), labels


class Mlp:
    """Parameters in fp32 and in the type of the products; one worker's forward and backward pass."""

    def __init__(self, ops, gen, dtype):
        self.ops, self.dtype = ops, dtype
        self.weights = [torch.randn(s, generator=gen, device="cuda") / s[1] ** 0.5 for s in LAYERS]
        self.biases = [torch.zeros(s[0], device="cuda") for s in LAYERS]
        self.refresh()

    def refresh(self):
        self.w = [t.to(self.dtype) for t in self.weights]
        self.b = [t.to(self.dtype) for t in self.biases]

    def forward(self, x):
        """(scores, what the backward pass needs: a checkpoint of every layer's input and of the activations' inputs)"""
        ops, n = self.ops, x.shape[0]
        inputs = [ops.save(x), B.Checkpoint.empty(n, HIDDEN), B.Checkpoint.empty(n, HIDDEN)]
        zs = [B.Checkpoint.empty(n, HIDDEN), B.Checkpoint.empty(n, HIDDEN), None]
        h1 = ops.forward(x, self.w[0], self.b[0], act=ACTS[0], save_z=zs[0], save_y=inputs[1])
        h2 = ops.forward(h1, self.w[1], self.b[1], h1, act=ACTS[1], save_z=zs[1], save_y=inputs[2])
        return ops.forward(h2, self.w[2], self.b[2]), (inputs, zs)

    def backward(self, dscores, kept, dw, db):
        """Gradients of the three weights and biases into dw and db (fp32)."""
        ops, (inputs, zs) = self.ops, kept
        dy, skip = dscores, None
        for l in (2, 1, 0):
            dz, _ = ops.activation_backward(dy, zs[l], ACTS[l], dbias=db[l])
            ops.weight_grad(dz, inputs[l], out=dw[l])
            if l == 0:
                break
            dx = ops.input_grad(dz, self.w[l])
            if l == 1:                                      # h2 = h1 + ...: h1's gradient has both ways
                dx += skip
            skip = dy = dx


def loss_and_gradient(scores, labels):
    p = torch.softmax(scores.float(), 1)
    picked = p.gather(1, labels[:, None])
    g = p.scatter_add(1, labels[:, None], -torch.ones_like(picked)) / len(labels)
    return -picked.log().mean(), g


def train(dtype=torch.float32, steps=30, workers=4, samples=256, rank=4, bits=8, eta=0.2, seed=0):
    """The losses, averaged over the workers, before each step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ops = B.LinearOps()
    net = Mlp(ops, gen, dtype)
    layers = B.layer_list(LAYERS, [s[0] for s in LAYERS])
    comp = B.Compressor(layers, rank, bits, bits, workers)
    for l, (rows, cols) in enumerate(LAYERS):
        comp.set_q(l, torch.randn((cols, min(rank, rows, cols)), generator=gen, device="cuda").cpu().numpy())
    grads = [[torch.empty(s, device="cuda") for s in LAYERS] + [torch.empty(s[0], device="cuda") for s in LAYERS] for _ in range(workers)]
    x, labels = make_data(workers, samples, gen)
    x = x.to(dtype)
    losses = []
    for _ in range(steps):
        total = torch.zeros((), device="cuda")
        for w in range(workers):
            scores, kept = net.forward(x[w])
            loss, g = loss_and_gradient(scores, labels[w])
            net.backward(g.to(dtype), kept, grads[w][:3], grads[w][3:])
            total += loss / workers
        comp.step_update(grads, net.weights + net.biases, eta)
        net.refresh()
        losses.append(total)
    comp.synchronize()
    out = [float(v) for v in losses]
    comp.close()
    ops.close()
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--type", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    for i, v in enumerate(train(torch.bfloat16 if a.type == "bf16" else torch.float32, a.steps)):
        print("step %3d  loss %.4f" % (i, v), flush=True)
