"""The longest sums of products of 8-bit rows that the call takes, close to 2^31, by every kernel that the rule gives them to."""
import pytest

from paper_2506_17974_amd import binding as B
from tests import int8_plan as ip
from tests.test_gpu_linear import U, _say, ops  # noqa: F401  (ops: the fixture)

K = B.INT8_MAX_COLS
# (samples, rows, kernel, four steps of operands in LDS, sum in parts)
CASES = [(1, 41, "token", False, False), (2, 5, "64", True, True), (67, 515, "64", True, True), (130, 4097, "128", False, True), (300, 2000, "128", True, True),
         (4100, 4097, "128", False, False), (700, 2000, "256", True, True), (2049, 4097, "256", True, False)]


@pytest.mark.skipif(ip.compiler() is None, reason="no C++ compiler")
def test_cases_take_the_kernels_they_are_for(tmp_path):
    for c, p in zip(CASES, ip.plans(ip.build(tmp_path), [(m, n, K) for m, n, *_ in CASES])):
        assert (p[0], p[1], p[2] > 1) == c[2:], (c, p)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,kernel,deep,parts", CASES)
def test_sums(ops, m, n, kernel, deep, parts):
    """Codes of -128 against -128 and 127: 128 (128 or -127) 131040, whose 19 digits fp32 holds, so that the outputs are equal.  Then random ones
    near the ends: 2 u of the rounded sum and of its product with the scale."""
    import torch
    _say("int8 largest sums", m, n, kernel, deep, parts)
    g = torch.Generator(device="cuda").manual_seed(m + n)
    x, w = torch.full((m, K), -128, dtype=torch.int8, device="cuda"), torch.full((n, K), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    xs, ws = torch.ones(m, device="cuda"), torch.full((n,), 2.0 ** -20, device="cuda")
    y = ops.int8_forward(B.RowCodes(x, xs, K), B.RowCodes(w, ws, K), dtype=torch.float32)
    want = torch.full((n,), 128.0 * 128 * K * 2.0 ** -20, device="cuda")
    want[1::2] = -128.0 * 127 * K * 2.0 ** -20
    assert (y == want).all()
    x.random_(-128, -119, generator=g)
    w[::2].random_(-128, -119, generator=g)
    w[1::2].random_(120, 128, generator=g)
    xs.uniform_(0.5, 1, generator=g)
    y = ops.int8_forward(B.RowCodes(x, xs, K), B.RowCodes(w, ws, K), dtype=torch.float32)
    want = torch.zeros((m, n), dtype=torch.float64, device="cuda")
    for k in range(0, K, 16384):
        want += torch.matmul(x[:, k:k + 16384].double(), w[:, k:k + 16384].double().t().contiguous())
    assert want.abs().min() > 1.8e9 and want.abs().max() < 2.0 ** 31
    want *= xs.double()[:, None] * 2.0 ** -20
    assert ((y.double() - want).abs() <= 2.01 * U * want.abs()).all()
