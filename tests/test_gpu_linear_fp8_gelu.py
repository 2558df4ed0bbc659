"""The GELU of astraea_gathered_linear_fp8 over every bf16 value, by both of its kernels (up to eight rows, and tiles)."""
import pytest
import torch

from paper_2506_05096_b200 import binding as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [7, 150])
@pytest.mark.parametrize("gate", [False, True])
def test_every_argument(rows, gate):
    """The products are zero, so that the GELU's argument is the bias: all 65536 bf16 codes, in an order that puts unlike ones side by side."""
    g = torch.Generator("cuda").manual_seed(rows)
    K, N_out = 128, 65536
    bias = torch.randperm(N_out, device="cuda", generator=g).to(torch.uint16).view(torch.bfloat16)
    xq, wq = torch.zeros(rows, K, device="cuda", dtype=torch.uint8), torch.zeros(N_out, K, device="cuda", dtype=torch.uint8)
    xs, ws = torch.ones(1, rows, device="cuda"), torch.ones(N_out // 128, 1, device="cuda")
    one = torch.ones(1, N_out, device="cuda", dtype=torch.bfloat16) if gate else None
    y = torch.empty(1, rows, N_out, device="cuda", dtype=torch.bfloat16)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, 1, 0, rows, rows, K)
    A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, bias, None, one, y, 1, rows, K, N_out, flags=A.LINEAR_GELU, workspace=work)
    A.astraea_poll_error(work)
    got, x = y[0].double(), bias.double()
    # what x Phi(x) gives: NaN at -infinity (0 * inf) and for NaN, infinity at +infinity
    odd = x.isnan() | (x == -float("inf"))
    assert torch.equal(got.isnan(), odd.expand(rows, -1))
    assert bool((got[:, x == float("inf")] == float("inf")).all())
    # Below -13 Phi is under 2^-120 and the result nothing, whatever the size of x; above 13 it is x
    low, high = (x < -13) & x.isfinite(), (x > 13) & x.isfinite()
    assert bool((got[:, low] == 0).all())
    assert torch.equal(got[:, high], x[high].expand(rows, -1))
    # Between them: Phi is within 7.5e-8 (half of erf's 1.5e-7) and four roundings of fp32, then one rounding to bf16 of the product
    mid = x.abs() <= 13
    phi = torch.special.ndtr(x[mid])
    off = x[mid].abs() * (7.5e-8 + 4 * 2.0 ** -24 * phi)
    excess = (got[:, mid] - x[mid] * phi).abs() - (off + 2.0 ** -8 * (x[mid].abs() * phi + off) + 2.0 ** -133)
    assert float(excess.max()) <= 0
