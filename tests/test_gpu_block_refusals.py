"""GPU tests of what the calls around the linear layer refuse; nothing that is refused is launched."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import _say, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu
M = N = K = 32


def _refused(code, call):
    with pytest.raises(B.LqsgdError) as e:
        call()
    assert e.value.code == code, str(e.value)


def test_outputs_over_inputs_and_each_other(ops):
    import torch
    _say("block overlaps")
    L, h = B.lib(), ops._h
    keep = [torch.zeros(M * K * 4, dtype=torch.uint8, device="cuda") for _ in range(16)]
    at = [t.data_ptr() for t in keep]
    last = lambda: L.lqsgd_linear_last_error(h).decode()  # noqa: E731

    def distinct_or_refused(call, names, outputs, inputs, allowed=()):
        args = dict(zip(names, at))
        assert call(**args) == B.OK, last()
        for o in outputs:
            for other in inputs + outputs:
                if other == o or (o, other) in allowed or (other, o) in allowed:
                    continue
                assert call(**dict(args, **{o: args[other]})) == B.EINVAL, (o, other)
                assert "output" in last()

    distinct_or_refused(lambda x, q, s: L.lqsgd_rows_save(h, 0, M, K, x, K, q, s), ("x", "q", "s"), ("q", "s"), ("x",))
    distinct_or_refused(lambda x, q, s: L.lqsgd_rows_load(h, 0, M, K, q, s, x, K), ("x", "q", "s"), ("x",), ("q", "s"))
    distinct_or_refused(lambda x, r, g, h_, y, rs, yc, ye, q, s: L.lqsgd_rms_norm(h, 0, M, K, 1e-6, x, K, r, K, g, h_, K, y, K, rs, yc, ye, q, s),
                        ("x", "r", "g", "h_", "y", "rs", "yc", "ye", "q", "s"), ("h_", "y", "rs", "yc", "ye", "q", "s"), ("x", "r", "g"),
                        (("h_", "x"), ("h_", "r")))
    distinct_or_refused(lambda dy, x, rs, g, dh, dx, dg: L.lqsgd_rms_norm_backward(h, 0, M, K, dy, K, x, K, None, None, rs, g, dh, K, dx, K, dg, 0),
                        ("dy", "x", "rs", "g", "dh", "dx", "dg"), ("dx", "dg"), ("dy", "x", "rs", "g", "dh"), (("dx", "dy"), ("dx", "dh")))
    distinct_or_refused(lambda dy, c, e, rs, dx, dg: L.lqsgd_rms_norm_backward(h, 0, M, K, dy, K, None, 0, c, e, rs, None, None, 0, dx, K, dg, 0),
                        ("dy", "c", "e", "rs", "dx", "dg"), ("dx", "dg"), ("dy", "c", "e", "rs"), (("dx", "dy"),))
    distinct_or_refused(lambda q, s, wq, ws, b, r, y: L.lqsgd_int8_forward(h, 0, 0, M, N, K, q, s, wq, ws, b, r, N, y, N),
                        ("q", "s", "wq", "ws", "b", "r", "y"), ("y",), ("q", "s", "wq", "ws", "b", "r"), (("y", "r"),))
    distinct_or_refused(lambda x, r, y, yc, ye, o: L.lqsgd_dropout(h, 0, M, K, 0.5, 1, 2, o, x, K, r, K, y, K, yc, ye),
                        ("x", "r", "y", "yc", "ye", "o"), ("y", "yc", "ye"), ("x", "r", "o"), (("y", "x"), ("y", "r")))
    torch.cuda.synchronize()


def test_arguments(ops):
    import torch
    _say("block arguments")
    L, h = B.lib(), ops._h
    t = torch.zeros(1 << 14, dtype=torch.uint8, device="cuda")
    p = [t.data_ptr() + 1024 * k for k in range(16)]

    def norm(type=0, samples=2, features=K, eps=1e-6, x=p[0], ldx=K, r=p[1], ldr=K, g=p[2], h_=p[3], ldh=K, y=p[4], ldy=K, rs=p[5], yc=None, ye=None, q=None, s=None):
        return L.lqsgd_rms_norm(h, type, samples, features, eps, x, ldx, r, ldr, g, h_, ldh, y, ldy, rs, yc, ye, q, s)

    assert norm() == B.OK and norm(samples=0, x=None) == B.OK
    for bad in (dict(type=3), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None, rs=None), dict(r=None),
                dict(x=p[0] + 2), dict(g=p[2] + 1), dict(rs=p[5] + 2), dict(yc=p[6]), dict(ye=p[6]), dict(yc=p[6] + 8, ye=p[7]), dict(q=p[6]), dict(s=p[6]),
                dict(q=p[6] + 4, s=p[7]), dict(q=p[6], s=p[7] + 2), dict(h_=p[0], ldx=K, ldh=K + 1), dict(h_=p[1], ldr=K + 1)):
        assert norm(**bad) == B.EINVAL, bad
    for bad in (dict(samples=-1), dict(samples=(1 << 30) + 1), dict(features=0), dict(features=(1 << 20) + 1), dict(ldx=K - 1), dict(ldr=K - 1), dict(ldh=K - 1),
                dict(ldy=(1 << 21) + 1)):
        assert norm(**bad) == B.ESHAPE, bad

    def back(type=0, samples=2, features=K, dy=p[0], lddy=K, x=p[1], ldh=K, c=None, e=None, rs=p[2], g=p[3], dh=p[4], lddh=K, dx=p[5], lddx=K, dg=p[6], acc=0):
        return L.lqsgd_rms_norm_backward(h, type, samples, features, dy, lddy, x, ldh, c, e, rs, g, dh, lddh, dx, lddx, dg, acc)

    assert back() == B.OK and back(x=None, c=p[7], e=p[8]) == B.OK and back(samples=0, dy=None, x=None, rs=None) == B.OK
    for bad in (dict(type=-1), dict(dy=None), dict(rs=None), dict(x=None), dict(c=p[7], e=p[8]), dict(x=None, c=p[7]), dict(x=None, c=p[7] + 8, e=p[8]),
                dict(dx=None, dg=None), dict(dg=p[6] + 2), dict(dx=p[0], lddx=K + 1), dict(dx=p[4], lddx=K + 1)):
        assert back(**bad) == B.EINVAL, bad
    for bad in (dict(samples=-1), dict(features=0), dict(lddy=K - 1), dict(ldh=K - 1), dict(lddh=K - 1), dict(lddx=K - 1)):
        assert back(**bad) == B.ESHAPE, bad

    def layer(type=0, act=0, samples=2, rows=8, cols=K, q=p[0], s=p[1], wq=p[2], ws=p[3], b=p[4], r=p[5], ldr=8, y=p[6], ldy=8):
        return L.lqsgd_int8_forward(h, type, act, samples, rows, cols, q, s, wq, ws, b, r, ldr, y, ldy)

    assert layer() == B.OK and layer(samples=0, q=None, s=None, y=None) == B.OK
    for bad in (dict(type=7), dict(act=4), dict(act=-1), dict(q=None), dict(s=None), dict(wq=None), dict(ws=None), dict(y=None), dict(q=p[0] + 8), dict(ws=p[3] + 2),
                dict(b=p[4] + 2), dict(y=p[5], ldr=9)):
        assert layer(**bad) == B.EINVAL, bad
    for bad in (dict(samples=-1), dict(rows=0), dict(cols=0), dict(cols=B.INT8_MAX_COLS + 1), dict(ldy=7), dict(ldr=7)):
        assert layer(**bad) == B.ESHAPE, bad

    def drop(type=0, samples=2, features=K, prob=0.5, more=None, x=p[0], ldx=K, r=p[1], ldr=K, y=p[2], ldy=K, yc=None, ye=None):
        return L.lqsgd_dropout(h, type, samples, features, prob, 1, 2, more, x, ldx, r, ldr, y, ldy, yc, ye)

    assert drop() == B.OK and drop(samples=0, x=None, y=None) == B.OK
    for bad in (dict(type=3), dict(prob=-0.1), dict(prob=1.1), dict(prob=float("nan")), dict(x=None), dict(y=None), dict(more=p[3] + 4), dict(yc=p[3]),
                dict(y=p[0], ldy=K + 1), dict(y=p[1], ldy=K + 1)):
        assert drop(**bad) == B.EINVAL, bad
    for bad in (dict(samples=-1), dict(features=0), dict(ldx=K - 1), dict(ldr=K - 1), dict(ldy=K - 1)):
        assert drop(**bad) == B.ESHAPE, bad
    for call in (lambda **a: L.lqsgd_rows_save(h, a.get("type", 0), a.get("n", 2), a.get("f", K), a.get("x", p[0]), a.get("ld", K), a.get("q", p[1]), a.get("s", p[2])),
                 lambda **a: L.lqsgd_rows_load(h, a.get("type", 0), a.get("n", 2), a.get("f", K), a.get("q", p[1]), a.get("s", p[2]), a.get("x", p[0]), a.get("ld", K))):
        assert call() == B.OK and call(n=0, x=None, q=None) == B.OK
        for bad in (dict(type=3), dict(x=None), dict(q=None), dict(s=None), dict(q=p[1] + 8), dict(s=p[2] + 2), dict(x=p[0] + 2)):
            assert call(**bad) == B.EINVAL, bad
        for bad in (dict(n=-1), dict(f=0), dict(ld=K - 1)):
            assert call(**bad) == B.ESHAPE, bad
    torch.cuda.synchronize()


def test_binding(ops):
    import torch
    _say("block binding")
    x, g = torch.randn(6, 40, device="cuda"), torch.randn(40, device="cuda")
    q, w = ops.quantize(x), ops.quantize(torch.randn(10, 40, device="cuda"))
    rstd = ops.rms_norm(x, want_rstd=True)[2]
    for call in (lambda: ops.rms_norm(x.cpu()), lambda: ops.rms_norm(x, g.half()), lambda: ops.rms_norm(x, g[:39]), lambda: ops.rms_norm(x, residual=x[:5]),
                 lambda: ops.rms_norm(x, residual=x.half()), lambda: ops.rms_norm(x.t()), lambda: ops.rms_norm(x, out=x.half()), lambda: ops.rms_norm(x.double()),
                 lambda: ops.rms_norm(x, rstd=rstd[:5]), lambda: ops.rms_norm(x, save_y=B.Checkpoint.empty(6, 41)),
                 lambda: ops.rms_norm(x, quantize_y=B.RowCodes.empty(5, 40)), lambda: ops.rms_norm(x, quantize_y=B.RowCodes.empty(6, 41)),
                 lambda: ops.rms_norm_backward(x, x[:5], rstd), lambda: ops.rms_norm_backward(x, x, rstd.double()), lambda: ops.rms_norm_backward(x, x, rstd, g, dh=x.half()),
                 lambda: ops.rms_norm_backward(x, x, rstd, dgain=g.half()), lambda: ops.rms_norm_backward(x, B.Checkpoint.empty(6, 39), rstd),
                 lambda: ops.int8_forward(q, ops.quantize(x[:, :39])), lambda: ops.int8_forward(q, w, bias=g[:10].half(), dtype=torch.float32),
                 lambda: ops.int8_forward(q, w, residual=x), lambda: ops.int8_forward(q, w, out=x),
                 lambda: ops.int8_forward(B.RowCodes(q.codes.t(), q.scales, 40), w), lambda: ops.int8_forward(B.RowCodes(q.codes, q.scales.double(), 40), w),
                 lambda: ops.dropout(x, 0.1, 1, residual=x.half()), lambda: ops.dropout(x, 0.1, 1, more_offset=rstd[:1]), lambda: ops.dropout(x, 0.1, 1, more_offset=3),
                 lambda: ops.dropout(x[0], 0.1, 1), lambda: ops.quantize(x.long()), lambda: ops.quantize(x, out=B.RowCodes.empty(6, 39)),
                 lambda: ops.dequantize(q, out=x[:5])):
        _refused(B.ESHAPE, call)
    for call in (lambda: ops.rms_norm(x, h=x.clone()), lambda: ops.rms_norm(x, want_y=False), lambda: ops.rms_norm(x, eps=-1.0), lambda: ops.rms_norm(x, out=x),
                 lambda: ops.rms_norm(x, quantize_y=B.Checkpoint.empty(6, 40)), lambda: ops.rms_norm_backward(x, x, rstd, accumulate=True),
                 lambda: ops.rms_norm_backward(x, x, rstd, want_dx=False, want_dgain=False), lambda: ops.int8_forward(x, w), lambda: ops.int8_forward(q, w, act="tanh"),
                 lambda: ops.int8_forward(q, w, dtype=torch.int8), lambda: ops.dropout(x, 1.5, 1), lambda: ops.dropout(x, 0.1, -1),
                 lambda: ops.dropout(x, 0.1, 1, 1 << 64), lambda: ops.dequantize(x), lambda: ops.dequantize(q, torch.float64)):
        _refused(B.EINVAL, call)


def test_another_device_or_stream_is_current():
    import torch
    _say("block on another device")
    mine = B.LinearOps()
    x = torch.ones((4, 8), device="cuda")
    q = mine.quantize(x)
    rstd = mine.rms_norm(x, want_rstd=True)[2]
    calls = [lambda: mine.quantize(x), lambda: mine.dequantize(q), lambda: mine.rms_norm(x), lambda: mine.rms_norm_backward(x, x, rstd),
             lambda: mine.int8_forward(q, q), lambda: mine.dropout(x, 0.5, 1)]
    asked = mine._current_device
    mine._current_device = lambda: mine.device.index + 1
    for call in calls:
        _refused(B.ESTATE, call)
    mine._current_device = asked
    with torch.cuda.stream(torch.cuda.Stream()):
        for call in calls:
            _refused(B.ESTATE, call)
    for call in calls:
        call()
    mine.close()
    for call in calls:
        _refused(B.ESTATE, call)


def test_tensors_that_require_a_gradient():
    import torch
    _say("block autograd")
    mine = B.LinearOps()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, r, dy = (torch.randn((5, 40), generator=g, device="cuda") for _ in range(3))
    gain = torch.randn(40, generator=g, device="cuda")
    b = torch.randn(40, generator=g, device="cuda")
    w = mine.quantize(torch.randn((40, 40), generator=g, device="cuda"))
    rstd = mine.rms_norm(x, want_rstd=True)[2]
    needs = lambda t: t.clone().requires_grad_()  # noqa: E731
    made = [*mine.rms_norm(needs(x), gain, r, want_rstd=True), *mine.rms_norm(x, needs(gain), r), *mine.rms_norm(x, gain, needs(r)),
            *mine.rms_norm_backward(needs(dy), x, rstd, gain), *mine.rms_norm_backward(dy, needs(x), rstd, gain), *mine.rms_norm_backward(dy, x, rstd, needs(gain)),
            *mine.rms_norm_backward(dy, x, rstd, gain, dh=needs(r)), mine.int8_forward(mine.quantize(x), w, needs(b)), mine.int8_forward(mine.quantize(x), w, b, needs(r)),
            mine.dropout(needs(x), 0.5, 1), mine.dropout(x, 0.5, 1, residual=needs(r))]
    for t in made:
        if t is None:
            continue
        assert t.requires_grad
        _refused(B.EINVAL, lambda: t.sum().backward())
    with torch.no_grad():
        assert not mine.dropout(needs(x), 0.5, 1).requires_grad and not mine.rms_norm(needs(x))[0].requires_grad
    assert not mine.dropout(x, 0.5, 1).requires_grad
    mine.close()
