"""Waits of the grouped products and of the norm's rings that give up: a call then ends with a timeout
or, where every wait was answered in time, with its result; the next call, with the
ordinary budget, gives the ordinary bits."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests.test_gpu_grouped import call as product
from tests.test_gpu_grouped import operands

pytestmark = pytest.mark.gpu
BUDGETS = [0, 1, 100, 300, 1000, 3000, 10000]


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def check(call):
    ref = [t.clone() for t in call()]
    assert C.ec2moe_last_device_error() == C.OK
    old = C.ec2moe_get_wait_budget()
    seen = set()
    for budget in BUDGETS * 2:
        try:
            C.ec2moe_set_wait_budget(budget)
            got = call()
            status = C.ec2moe_last_device_error()
        finally:
            C.ec2moe_set_wait_budget(old)
        assert status in (C.OK, C.ERR_TIMEOUT)
        seen.add(status)
        if status == C.OK:
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
        got = call()
        assert C.ec2moe_last_device_error() == C.OK and all(torch.equal(a, b) for a, b in zip(got, ref))
    return seen


# tails in every group; one block per tile and many; split sums; several tiles per pair
@pytest.mark.parametrize("form", ["fwd", "dgrad", "wgrad"])
@pytest.mark.parametrize("offsets,N,K,out", [([0, 33, 33, 250, 701], 264, 520, C.BF16), ([0, 700], 512, 2048, C.F32),
                                             ([0, 9, 20, 40], 4096, 2048, C.F32), ([0, 3001, 6002], 1024, 4096, C.BF16)])
def test_products(form, offsets, N, K, out):
    G, rows = len(offsets) - 1, offsets[-1]
    X, W = operands(form, rows, N, K, G)
    assert C.ERR_TIMEOUT in check(lambda: [product(form, X, W, offsets, G, rows, N, K, out)])


# long calls, whose rings have to wait for memory; short ones, whose rows may be there before they are asked for
@pytest.mark.parametrize("rows,cols,waits", [(40000, 2048, True), (20000, 4096, True), (1000, 768, False), (400, 16384, False)])
def test_norm(rows, cols, waits):
    x, dy = (torch.randn(rows, cols, device="cuda").to(torch.bfloat16) for _ in range(2))
    w, rstd, dw = torch.ones(cols, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(C.ec2moe_rmsnorm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")

    def forward():
        C.ec2moe_rmsnorm(C.BF16, C.BF16, rows, cols, cols, x, None, w, 1e-5, None, rstd, y)
        return [y, rstd]

    assert C.ERR_TIMEOUT in check(forward) or not waits

    def backward():
        C.ec2moe_rmsnorm_backward(C.BF16, C.BF16, rows, cols, cols, dy, x, rstd, w, None, dx, dw, ws, ws.numel())
        return [dx, dw]

    assert C.ERR_TIMEOUT in check(backward) or not waits
