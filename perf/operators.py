"""The operators of a linear layer that trains with 8-bit activation checkpoints: the forward product with bias, activation
and residual, the checkpoints, and the three parts of the backward pass that end in the gradients the compressor takes.

x is samples x cols, w rows x cols (rows = output features), y samples x rows:

    linear               z = x w^T + bias;  y = act(z) + residual;  z and y may be kept in 8 bits as well
    checkpoint           x -> 8 bits -> x^
    activation_backward  dz = dy act'(z^);  dbias = sum over samples of dy act'(z^)
    input_grad           dx = dz w
    weight_grad          dw = dz^T x^

A checkpoint holds a tensor's rows in groups of 32 features: a group shares a power of two 2^e, e the smallest integer with
absmax / 2^e < 127.5 (bounded to what the type can hold), and a value v is kept as the nearest integer to v / 2^e.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

GROUP = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EXPONENTS = {"f32": (-126, 121), "bf16": (-126, 121), "f16": (-24, 9)}   # least and largest e of a type's checkpoints
ACTS = ("none", "relu", "gelu", "silu")


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _case(name, op, samples, cols, rows=0, dtype="bf16", act="none", bias=False, residual=False, save="", grad="f32", dist="normal"):
    c = {"op": op, "samples": samples, "rows": rows, "cols": cols, "dtype": dtype, "act": act, "bias": bias, "residual": residual,
         "save": save, "grad": grad, "dist": dist}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through the widening projection of a language model's block: the weight is read once, nothing else counts
        _case("linear_token_bf16", "linear", 1, 4096, 11008, act="silu", bias=True),
        # a batch of images through the small CNN's hidden layer, in 32 bits, z kept for the backward pass
        _case("linear_cnn_f32", "linear", 64, 3136, 1024, dtype="f32", act="relu", bias=True, save="z"),
        # odd sizes, 16-bit floats with a residual: a small hidden layer on concatenated features
        _case("linear_ragged_f16", "linear", 300, 513, 257, dtype="f16", act="gelu", bias=True, residual=True),
        # training: a language model's widening projection, both checkpoints written beside y
        _case("linear_llm_bf16", "linear", 4096, 4096, 11008, act="gelu", bias=True, save="zy", dist="outliers"),
        # what a layer keeps of its input: a small ragged one in 32 bits, and a language model's
        _case("checkpoint_ragged_f32", "checkpoint", 129, 1155, dtype="f32", dist="relu"),
        _case("checkpoint_llm_bf16", "checkpoint", 8192, 4096, dist="outliers"),
        # the activation's backward: the small CNN's in 32 bits, a language model's in 16
        _case("act_backward_cnn_f32", "activation_backward", 64, 1024, dtype="f32", act="relu"),
        _case("act_backward_llm_bf16", "activation_backward", 4096, 11008, act="gelu"),
        # the gradients: a ragged weight's in half floats, a language model's as the compressor takes it, and that of the input
        _case("weight_grad_ragged_f16", "weight_grad", 300, 2049, 1000, dtype="f16"),
        _case("weight_grad_llm_bf16", "weight_grad", 8192, 4096, 4096, dist="outliers"),
        _case("input_grad_llm_bf16", "input_grad", 4096, 4096, 11008),
        # a wide square layer trained in 32 bits
        _case("input_grad_8192_f32", "input_grad", 2048, 8192, 8192, dtype="f32"),
    ]


MOST_FLOPS = {"f32": 2.0 * 2048 * 8192 * 8192, "bf16": 2.0 * 4096 * 4096 * 11008, "f16": 2.0 * 4096 * 4096 * 11008}
MOST_VALUES = 4096 * 11008


def draw(rng):
    """Samples from one to a long batch, widths from small heads to a language model's, of any residue, every type and option."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width():
        n, kind = log_int(16, 11008), rng.random()
        return max(16, n // 64 * 64) if kind < 0.5 else max(16, n // 8 * 8) if kind < 0.75 else n

    op = rng.choice(("linear", "linear", "linear", "checkpoint", "activation_backward", "input_grad", "weight_grad", "weight_grad"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32", "f32", "f16"))
    samples, rows, cols = log_int(1, 8192), width(), width()
    if op in ("checkpoint", "activation_backward"):
        samples = max(1, min(samples, MOST_VALUES // cols))
        return _case(None, op, samples, cols, dtype=dtype, act=rng.choice(ACTS[1:]) if op == "activation_backward" else "none",
                     dist=rng.choice(("normal", "outliers", "relu")) if op == "checkpoint" else "normal")
    samples = max(1, min(samples, int(MOST_FLOPS[dtype] / (2.0 * rows * cols)), MOST_VALUES // max(rows, cols)))
    if op == "linear":
        return _case(None, op, samples, cols, rows, dtype, rng.choice(ACTS), rng.random() < 0.7, rng.random() < 0.3,
                     rng.choice(("", "", "z", "zy")), dist=rng.choice(("normal", "outliers", "relu")))
    return _case(None, op, samples, cols, rows, dtype, grad="bf16" if op == "weight_grad" and dtype == "bf16" and rng.random() < 0.3 else "f32",
                 dist=rng.choice(("normal", "outliers", "relu")) if op == "weight_grad" else "normal")


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _values(shape, gen, dist="normal", scale=1.0):
    x = torch.randn(shape, generator=gen, device="cuda")
    if dist == "relu":
        x.clamp_(min=0)
    elif dist == "outliers":             # a few features are large in every sample
        x.mul_(torch.rand(shape[-1], generator=gen, device="cuda").lt(0.01).float().mul_(19.0).add_(1.0))
    return x.mul_(scale)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 29)
    T, M, N, K = TYPES[case["dtype"]], case["samples"], case["rows"], case["cols"]
    s, op = {"case": case}, case["op"]
    if op == "linear":
        s["x"] = _values((M, K), gen, case["dist"]).to(T)
        s["w"] = _values((N, K), gen, scale=1.0 / math.sqrt(K)).to(T)
        s["bias"] = _values((N,), gen, scale=0.3).to(T) if case["bias"] else None
        s["residual"] = _values((M, N), gen).to(T) if case["residual"] else None
    elif op == "checkpoint":
        s["x"] = _values((M, K), gen, case["dist"]).to(T)
    elif op == "activation_backward":
        s["dy"] = _values((M, K), gen, scale=1e-2).to(T)
        s["codes"], s["exponents"] = _quantise(_values((M, K), gen, scale=1.5), case["dtype"])
    elif op == "input_grad":
        s["dz"] = _values((M, N), gen, scale=1e-2).to(T)
        s["w"] = _values((N, K), gen, scale=1.0 / math.sqrt(K)).to(T)
    else:
        s["dz"] = _values((M, N), gen, scale=1e-2).to(T)
        s["codes"], s["exponents"] = _quantise(_values((M, K), gen, case["dist"]).to(T).float(), case["dtype"])
    return s


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _quantise(v, dtype):
    """(codes: int8, samples x the features rounded up to whole groups; exponents: uint8, e + 127 of each group, 255 where
    the group holds a value that is not finite)."""
    lo, hi = EXPONENTS[dtype]
    M, K = v.shape
    groups = -(-K // GROUP)
    p = torch.zeros((M, groups * GROUP), device=v.device)
    p[:, :K] = v
    p = p.view(M, groups, GROUP)
    absmax = p.abs().amax(-1)
    e = (((absmax.view(torch.int32) + 0x10000) >> 23) - 133).clamp(lo, hi)     # the carry is the step past 127.5 / 64
    step = ((127 - e) << 23).view(torch.float32)                               # 2^-e
    q = torch.round(p * step[..., None]).clamp(-127, 127)
    bad = ~torch.isfinite(p).all(-1)
    q = torch.where(bad[..., None], torch.zeros_like(q), q)
    e = torch.where(bad, torch.full_like(e, 128), e)
    return q.to(torch.int8).view(M, groups * GROUP), (e + 127).to(torch.uint8)


def _dequantise(codes, exponents, features):
    e = exponents.to(torch.int32)
    scale = torch.where(e == 255, torch.full(e.shape, math.nan, device=e.device), (e << 23).view(torch.float32))
    M, groups = exponents.shape
    return (codes.view(M, groups, GROUP).float() * scale[..., None]).view(M, groups * GROUP)[:, :features]


def _activate(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).float() + (z - z)         # a value that is not a number has no slope
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    T = TYPES[case["dtype"]]
    if op == "linear":
        z = s["x"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _activate(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(T)}
        kept = torch.float16 if T == torch.float16 else torch.bfloat16
        if "z" in case["save"]:
            out["z_kept"] = _dequantise(*_quantise(z, case["dtype"]), case["rows"]).to(kept)
        if "y" in case["save"]:
            out["y_kept"] = _dequantise(*_quantise(out["y"].float(), case["dtype"]), case["rows"]).to(kept)
        return out
    if op == "checkpoint":
        return {"x_kept": _dequantise(*_quantise(s["x"].float(), case["dtype"]), case["cols"]).to(T)}
    if op == "activation_backward":
        dz = s["dy"].float() * _slope(_dequantise(s["codes"], s["exponents"], case["cols"]), case["act"])
        return {"dz": dz.to(T), "dbias": dz.sum(0)}
    if op == "input_grad":
        return {"dx": (s["dz"].float() @ s["w"].float()).to(T)}
    dw = s["dz"].float().t() @ _dequantise(s["codes"], s["exponents"], case["cols"])
    return {"dw": dw.to(TYPES[case["grad"]])}


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _binding():
    from paper_2506_17974_amd import binding
    return binding


@functools.lru_cache(maxsize=None)
def _ops():
    return _binding().LinearOps()


def _own(s):
    B, ops = _binding(), _ops()
    case, op = s["case"], s["case"]["op"]
    if op == "linear":
        M, N = case["samples"], case["rows"]
        zk = B.Checkpoint.empty(M, N) if "z" in case["save"] else None
        yk = B.Checkpoint.empty(M, N) if "y" in case["save"] else None
        out = {"y": ops.forward(s["x"], s["w"], s["bias"], s["residual"], act=case["act"], save_z=zk, save_y=yk)}
        kept = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
        if zk is not None:
            out["z_kept"] = ops.load(zk, kept)
        if yk is not None:
            out["y_kept"] = ops.load(yk, kept)
        return out
    if op == "checkpoint":
        return {"x_kept": ops.load(ops.save(s["x"]), TYPES[case["dtype"]])}
    if op == "activation_backward":
        dz, db = ops.activation_backward(s["dy"], B.Checkpoint(s["codes"], s["exponents"], case["cols"]), act=case["act"])
        return {"dz": dz, "dbias": db}
    if op == "input_grad":
        return {"dx": ops.input_grad(s["dz"], s["w"])}
    return {"dw": ops.weight_grad(s["dz"], B.Checkpoint(s["codes"], s["exponents"], case["cols"]), dtype=TYPES[case["grad"]])}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    M, N, K, s = case["samples"], case["rows"], case["cols"], SIZE[case["dtype"]]
    held = 1.0 + 1.0 / GROUP
    if case["op"] == "linear":
        n = s * (M * K + N * K + M * N) + s * N * case["bias"] + s * M * N * case["residual"]
        n += len(case["save"]) * M * N * (2 * held + 2)          # written, and read again to be returned as values
        return {"bytes": n, "flops": 2.0 * M * N * K}
    if case["op"] == "checkpoint":
        return {"bytes": M * K * (2 * s + 2 * held), "flops": 2.0 * M * K}
    if case["op"] == "activation_backward":
        return {"bytes": M * K * (2 * s + held) + 4 * K, "flops": 2.0 * M * K}
    if case["op"] == "input_grad":
        return {"bytes": s * (M * N + N * K + M * K), "flops": 2.0 * M * N * K}
    return {"bytes": s * M * N + held * M * K + SIZE[case["grad"]] * N * K, "flops": 2.0 * M * N * K}


# ---------------------------------------------------------------------------
# the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _held(v, dtype):
    """The values a checkpoint of v stands for: v in units of a power of two that takes the group's largest value to (63.75, 127.5)."""
    v = v.double()
    lo, hi = EXPONENTS[dtype]
    M, K = v.shape
    g = torch.nn.functional.pad(v, (0, -K % GROUP)).reshape(M, -1, GROUP)
    mantissa, power = torch.frexp(g.abs().amax(-1))                       # 1/2 <= mantissa < 1
    e = power.to(torch.int64) - 7 + (mantissa * 128 >= 127.5)
    e = torch.where(mantissa == 0, torch.full_like(e, lo), e).clamp(lo, hi)[..., None]
    unit = ((e + 1023) << 52).view(torch.float64)
    q = torch.clamp(torch.round(g / unit), -127, 127) * unit
    return q.reshape(M, -1)[:, :K]


def _value(codes, exponents, features):
    unit = ((exponents.long() + 1023 - 127) << 52).view(torch.float64)
    return (codes.double() * unit.repeat_interleave(GROUP, 1))[:, :features]


def exact(case, seed):
    s, op, act = prepare(case, seed), case["op"], case["act"]
    if op == "linear":
        z = torch.matmul(s["x"].double(), s["w"].double().t().contiguous())
        if case["bias"]:
            z += s["bias"].double()
        if act == "relu":
            y = z.clamp(min=0)
        elif act == "gelu":
            y = z * torch.special.erfc(z / -math.sqrt(2)) / 2
        elif act == "silu":
            y = z * torch.sigmoid(z)
        else:
            y = z
        out = {"y": y + s["residual"].double() if case["residual"] else y}
        return dict(out, **{k + "_kept": None for k in case["save"]})     # a value at the middle of two codes may take either
    if op == "checkpoint":
        return {"x_kept": _held(s["x"], case["dtype"])}
    if op == "activation_backward":
        z = _value(s["codes"], s["exponents"], case["cols"])
        if act == "relu":
            slope = torch.heaviside(z, torch.zeros_like(z))
        elif act == "gelu":
            slope = torch.special.erfc(z / -math.sqrt(2)) / 2 + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
        else:
            slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        dz = slope * s["dy"].double()
        return {"dz": dz, "dbias": dz.sum(0)}
    if op == "input_grad":
        return {"dx": torch.matmul(s["dz"].double(), s["w"].double())}
    return {"dw": torch.matmul(s["dz"].double().t().contiguous(), _value(s["codes"], s["exponents"], case["cols"]))}
