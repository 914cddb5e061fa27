"""Hidden rows of SwiGLU experts: identity weights show them.  They are the exact
activation's, rounded to e4m3, except where that lies within the errors of a tie.

With u = q s (exact products by 1, one rounding of q s), silu(u) u has, relative to
itself: e^-u by the hardware's exponential (2^-22) of an argument rounded to 2^-24 |u|,
1 + e^-u, a division of 2 units in the last place, the product and u's own rounding
twice: below 2^-22 + 8 2^-24 + 2^-22 + 4 2^-24 = 1.2e-6 for |u| <= 8.4.  The block's scale
comes from the largest value with the same error, and takes three further roundings:
together below 2.6e-6."""
import numpy as np
import pytest
import torch

from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# few rows (partial sums and the activation in a kernel of its own), single tiles, pairs
@pytest.mark.parametrize("T", [8, 200, 4096])
@pytest.mark.parametrize("n", [128, 384])
def test_hidden_rows_are_the_exact_activation_rounded(T, n):
    rng = np.random.default_rng(T + n)
    q = rng.integers(0, 255, size=(T, n), dtype=np.uint8)
    q[(q & 0x7F) == 0x7F] = 0
    s = np.exp(rng.uniform(-9, -4, size=(T, n // 128))).astype(np.float32)
    one = cuda(np.where(np.eye(n), 0x38, 0).astype(np.uint8))
    scale = torch.ones(n // 128, n // 128, device="cuda")
    w = C.make_fp8_weights(W1=one, S1=scale, W3=one, S3=scale, W2=one, S2=scale)
    desc = C.make_desc(T=T, d=n, E=1, d_ff=n, k=1, act=C.SWIGLU, dtype=C.F32)
    wsb = C.ec2moe_experts_fp8_workspace_size(desc)
    out = torch.empty(T, n, device="cuda")
    C.ec2moe_experts_fp8(desc, cuda(q), cuda(s), cuda(np.array([0, T], np.int32)), w, torch.ones(T, 1, device="cuda"),
                         torch.arange(T, dtype=torch.int32, device="cuda"), out,
                         torch.empty(wsb, dtype=torch.uint8, device="cuda"), wsb)
    assert C.ec2moe_last_device_error() == C.OK
    u = orc.e4m3_decode(q) * np.repeat(s.astype(np.float64), 128, 1)
    h = orc.silu(u) * u
    to_grid = np.repeat(448.0 / np.maximum(np.abs(h).reshape(T, -1, 128).max(2), 2.0 ** -96), 128, 1)
    r = h * to_grid
    codes = np.arange(256, dtype=np.uint8)
    grid = np.unique(orc.e4m3_decode(codes[(codes & 0x7F) != 0x7F]))
    at = np.clip(np.searchsorted(grid, r), 1, len(grid) - 1)
    lo, hi = grid[at - 1], grid[at]
    tie = (lo + hi) / 2
    sure = np.abs(r - tie) > 2.6e-6 * np.abs(r) + 1e-12
    want = np.where(r < tie, lo, hi)
    got = out.double().cpu().numpy() * to_grid
    assert sure.mean() > 0.99
    assert (np.abs(got - want)[sure] <= 1e-5 * np.abs(want)[sure] + 1e-12).all()
