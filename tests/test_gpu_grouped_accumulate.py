"""Weights' gradients that are added to: a group without rows leaves its part as it was, bit for bit."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests.test_gpu_grouped import call, operands

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


# one range; ranges of a cluster (few tiles, long sums); ranges in the workspace
@pytest.mark.parametrize("G,rows,N,K", [(8, 700, 1024, 2048), (2, 8191, 512, 1024), (2, 16000, 512, 4096), (1, 8191, 512, 4096),
                                        (4, 20000, 256, 256)])
def test_groups_without_rows(G, rows, N, K):
    offsets = [0] * G + [rows]  # all rows are the last group's
    X, W = operands("wgrad", rows, N, K, G, seed=8)
    g = torch.Generator(device="cuda").manual_seed(1)
    before = torch.randn(G, N, K, generator=g, device="cuda")
    before[before.abs() < 0.1] = -0.0
    sums = call("wgrad", X, W, offsets, G, rows, N, K, C.F32)
    got = call("wgrad", X, W, offsets, G, rows, N, K, C.F32, accumulate=1, into=before.clone())
    assert C.ec2moe_last_device_error() == C.OK
    assert torch.equal(got[-1], before[-1] + sums[-1])
    assert torch.equal(got[:-1].view(torch.int32), before[:-1].view(torch.int32))
    none = call("wgrad", X, W, [rows] * (G + 1), G, rows, N, K, C.F32, accumulate=1, into=before.clone())
    assert torch.equal(none.view(torch.int32), before.view(torch.int32))
