"""The norm's longer calls with the sum in the place of X or of the residual: rows are fetched ahead of those stored."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


@pytest.mark.parametrize("rows,cols", [(1200, 2048), (5003, 768), (700, 9000), (20000, 4096), (311, 16384)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sum_in_an_operands_place(rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    code = C.BF16 if dtype == torch.bfloat16 else C.F32
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")

    def call(a, b, into):
        Y, rstd = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(rows, device="cuda")
        C.ec2moe_rmsnorm(code, code, rows, cols, cols, a, b, w, 1e-5, into, rstd, Y)
        return into, rstd, Y

    want = call(x, r, torch.empty_like(x))
    assert torch.equal(want[0], (x.float() + r.float()).to(dtype))
    for place in range(2):
        a, b = x.clone(), r.clone()
        got = call(a, b, (a, b)[place])
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    a = x.clone()
    both = call(a, a, a)  # one tensor in all three places
    assert torch.equal(both[0], (2 * x.float()).to(dtype))
    assert C.ec2moe_last_device_error() == C.OK
