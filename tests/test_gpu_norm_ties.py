"""The norm's 8-bit rows at e4m3's ties, in the normal and the subnormal range.

What a value is rounded from is 448 |h w| over the block's largest |h w|, the row's rstd being in
both.  The reference decides each by exact products in 64 bits: 48 bits of h w times 448 = 7 2^6
(51 bits), and 48 bits of the largest times a tie's 5 (53 bits).
"""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def ties():
    """Every value half way between two neighbours of e4m3, up to 432."""
    below = [(2 * n + 1) * 2.0 ** -10 for n in range(8)]
    normal = [(17 + 2 * n) / 16 * 2.0 ** e for e in range(-6, 9) for n in range(8)]
    return torch.tensor(below + [t for t in normal if t < 448], dtype=torch.float64, device="cuda")


def definition(h, w):
    """e4m3 values of h w, in blocks of 128 columns whose largest magnitude becomes 448."""
    p = (h.double() * w.double()).view(h.shape[0], -1, 128)
    num, most = 448 * p.abs(), p.abs().amax(2, keepdim=True)
    q = num / most
    step = torch.exp2(torch.floor(torch.log2(q.clamp_min(2.0 ** -6))) - 3)
    n = torch.floor(q / step)
    tie = (n + 0.5) * step * most
    up = (num > tie) | ((num == tie) & (n % 2 == 1))
    return (torch.where(up, n + 1, n) * step * torch.sign(p)).view(h.shape)


def rows8(x, weight):
    rows, cols = x.shape
    code = C.BF16 if x.dtype == BF else C.F32
    Q, S = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, cols // 128, device="cuda")
    C.ec2moe_rmsnorm(code, code, rows, cols, cols, x, None, weight, 1e-5, None, None, None, Q, S)
    return Q.to(F32).double()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [80, 1200])
def test_ties_go_to_the_even_neighbour(rows, dtype):
    """Blocks with 7 2^k as their largest and every tie in it, exactly."""
    t = ties()
    g = torch.Generator(device="cuda").manual_seed(rows)
    block = torch.cat([torch.tensor([448.0, 0.0], dtype=torch.float64, device="cuda"), t])
    assert block.numel() == 128
    order = torch.stack([torch.randperm(128, generator=g, device="cuda") for _ in range(2 * rows)])
    sign = torch.randint(0, 2, (2 * rows, 128), generator=g, device="cuda") * 2 - 1
    k = torch.randint(-20, 21, (2 * rows, 1), generator=g, device="cuda").double()
    x64 = (block[order] * sign * torch.exp2(k - 6)).view(rows, 256)
    x = x64.to(dtype)
    assert torch.equal(x.double(), x64)
    ones = torch.ones(256, device="cuda")
    got, want = rows8(x, None), definition(x, ones)
    assert torch.equal(got, want), (int((got != want).sum()), want[got != want].unique().tolist()[:20])


@pytest.mark.parametrize("rows,cols", [(250, 2048), (3000, 1024)])
@pytest.mark.parametrize("weighted", [False, True])
def test_values_beside_ties(rows, cols, weighted):
    """fp32 values within 8 units of their last place of a tie, of a block's largest of any mantissa."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    t = ties()
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).abs() + 0.05 if weighted else torch.ones(cols, device="cuda")
    n = rows * (cols // 128)
    most = (1 + torch.rand(n, 1, generator=g, device="cuda", dtype=torch.float64)) * w.double().max()
    pick = t[torch.randint(0, t.numel(), (n, 128), generator=g, device="cuda")]
    units = torch.randint(-8, 9, (n, 128), generator=g, device="cuda")
    wb = w.double().view(1, -1, 128).expand(rows, -1, -1).reshape(n, 128)
    h = (pick * most / (448 * wb)).float()
    h = (h.view(torch.int32) + units.int()).view(F32)
    h[:, 5] = (most[:, 0] / wb[:, 5]).float()
    x = h.view(rows, cols)
    got, want = rows8(x, w if weighted else None), definition(x, w)
    assert torch.equal(got, want), (int((got != want).sum()), want[got != want].unique().tolist()[:20])
