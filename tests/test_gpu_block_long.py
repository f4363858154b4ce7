"""GPU tests of the norm's backward pass where a workgroup takes several rows, in every kernel, and of large tensors from a checkpoint.

Bounds as in test_gpu_block.py, u = 2^-24: along (the mean of v h rstd) is a sum of `features` terms in fp32, dgain one of `samples`; 4 roundings of each of
dx's terms; and the output's own."""
import pytest

from paper_2506_17974_amd import binding as B
from tests.test_gpu_linear import HALF_ULP, TYPES, U, _say, _t, ops  # noqa: F401  (ops: the fixture)

pytestmark = pytest.mark.gpu

# (samples, features): wavefronts a row of 512, 768 and 1024 threads' kernels, with and without a piece cut by the row's end, several rows and a last
# one alone to a workgroup, and rows in two kernels, by runs of several and a last one of one
SEVERAL = [(601, 1500), (601, 3001), (601, 4608), (601, 7001), (601, 8192), (601, 11003), (601, 14001), (601, 16384), (501, 17003), (130, 40000)]
# more than 2^24 values: inputs past the caches
LARGE = [(35000, 481), (8200, 2049), (4200, 4099), (3300, 5090), (2400, 7003), (1600, 11003), (1200, 14003), (1060, 16001), (1000, 17003)]

# to either side of where one kernel makes dgain: a run alone, up to 64 runs of four rows, one row or more to a workgroup
FEW = [(1, 9), (4, 1024), (5, 1024), (64, 1024), (65, 1024), (256, 64), (257, 64), (260, 24), (512, 32), (1, 1025), (2, 1025), (1, 4097), (2, 4097), (1, 16384), (2, 16384)]


def _check(ops, kind, samples, features, source):
    import torch
    _say("norm backward", kind, samples, features, source)
    gen = torch.Generator(device="cuda").manual_seed(samples + features)

    def new(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(_t(kind))

    x, dy, dh, gain = new(samples, features), new(samples, features, scale=0.1), new(samples, features, scale=0.1), 1 + new(features, scale=0.3)
    rstd = ops.rms_norm(x, want_rstd=True, want_y=False)[2]
    if source == "checkpoint":
        x = ops.save(x)
    before = torch.randn(features, generator=gen, device="cuda")
    dgain = before.clone()
    dx, _ = ops.rms_norm_backward(dy, x, rstd, gain, dh=dh, dgain=dgain, accumulate=True)
    h = (ops.load(x, torch.float32) if source == "checkpoint" else x).double()
    r = rstd.double()[:, None]
    v, xh = dy.double() * gain.double(), h * r
    want = r * (v - xh * (v * xh).mean(1, keepdim=True)) + dh.double()
    along = (v * xh).abs().mean(1, keepdim=True)
    rel, least = HALF_ULP[kind]
    tol = (r * xh).abs() * along * U * (8 + 4 * features ** 0.5) + 4 * U * (r * (v.abs() + xh.abs() * along) + dh.double().abs()) + rel * want.abs() + least
    bad = ~((dx.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    terms = dy.double() * xh
    total = terms.sum(0) + before.double()
    bad = ~((dgain.double() - total).abs() <= U * terms.abs().sum(0) * (8 + 4 * samples ** 0.5) + U * total.abs())
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    # the same bits again, and in place
    again = torch.empty_like(dgain)
    got = ops.rms_norm_backward(dy, x, rstd, gain, dh=dh, dx=dy, dgain=again)
    assert got[0] is dy and torch.equal(dy, dx)
    assert ((again.double() - terms.sum(0)).abs() <= U * terms.abs().sum(0) * (8 + 4 * samples ** 0.5)).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", SEVERAL)
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_several_rows_to_a_workgroup(ops, kind, samples, features, source):
    assert samples * features <= 1 << 24
    _check(ops, kind, samples, features, source)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", LARGE)
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_past_the_caches(ops, kind, samples, features, source):
    assert samples * features > 1 << 24
    _check(ops, kind, samples, features, source)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("samples,features", FEW)
@pytest.mark.parametrize("source", ["tensor", "checkpoint"])
def test_few_runs(ops, kind, samples, features, source):
    for _ in range(2):                                        # whoever joins the runs leaves the count as it was
        _check(ops, kind, samples, features, source)
