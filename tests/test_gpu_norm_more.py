"""The norm's longer calls on narrow rows, and its gradient in the place of each operand."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests import test_gpu_norm as norm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


@pytest.mark.parametrize("rows,cols", [(5000, 8), (40001, 16), (1000, 24), (3000, 272)])
@pytest.mark.parametrize("dtype,y_dtype", [(BF, BF), (F32, F32)])
def test_narrow_rows(rows, cols, dtype, y_dtype):
    norm.test_forward(rows, cols, dtype, y_dtype, True)
    norm.test_backward(rows, cols, dtype, y_dtype, True)


@pytest.mark.parametrize("rows,cols", [(3, 24), (700, 4096), (5003, 768), (311, 16384)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradient_in_an_operands_place(rows, cols, dtype):
    code = C.BF16 if dtype == BF else C.F32
    dy, h, dh = (norm.rand(rows, cols, dtype=dtype, seed=s).contiguous() for s in range(3))
    w, rstd = 1 + 0.3 * norm.rand(cols, seed=3), torch.rand(rows, device="cuda") + 0.5
    ws = torch.empty(C.ec2moe_rmsnorm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")

    def call(place):
        t = [dy.clone(), h.clone(), dh.clone(), torch.empty_like(h)]
        dw = torch.empty(cols, device="cuda")
        C.ec2moe_rmsnorm_backward(code, code, rows, cols, cols, t[0], t[1], rstd, w, t[2], t[place], dw, ws, ws.numel())
        return t[place], dw

    want = call(3)
    for place in range(3):
        assert all(torch.equal(a, b) for a, b in zip(call(place), want)), place
    assert C.ec2moe_last_device_error() == C.OK
