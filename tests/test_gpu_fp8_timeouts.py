"""Waits that give up, whichever warp's it is: short budgets on calls whose copies are all
on their way before anything is waited for, and on longer ones.  A call then ends with a
timeout or, where every wait was answered in time, with its result; the next call, with
the ordinary budget, gives the ordinary bits (nothing of the call before lands in its
memory)."""
import numpy as np
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu
BUDGETS = [0, 1, 100, 300, 1000, 3000, 10000]


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def check(call):
    """call() -> results; status after it."""
    ref = call().clone()
    assert C.ec2moe_last_device_error() == C.OK
    old = C.ec2moe_get_wait_budget()
    for budget in BUDGETS * 2:
        try:
            C.ec2moe_set_wait_budget(budget)
            got = call()
            status = C.ec2moe_last_device_error()
        finally:
            C.ec2moe_set_wait_budget(old)
        assert status in (C.OK, C.ERR_TIMEOUT)
        if status == C.OK:
            assert torch.equal(got, ref)
        got = call()
        assert C.ec2moe_last_device_error() == C.OK and torch.equal(got, ref)


# clusters of 8, 4, 2 CTAs with one or a few blocks each; whole tiles; wide rows
@pytest.mark.parametrize("T,d,E,K", [(100, 512, 16, 4), (1, 2048, 64, 8), (2000, 256, 64, 8), (6000, 512, 8, 1), (30000, 512, 112, 16)])
def test_gate_logits(T, d, E, K):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    X = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    W = [torch.randn(n, d, generator=g, device="cuda") for n in (E, K)]
    b = [torch.randn(n, generator=g, device="cuda") for n in (E, K)]
    desc = C.make_desc(T=T, d=d, E=E, d_ff=0, k=1, n_groups=K)
    wsb = C.ec2moe_gate_logits_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.empty(T, E + (K if K > 1 else 0), device="cuda")

    def call():
        out.fill_(3.0)
        C.ec2moe_gate_logits(desc, X, W[0], b[0], W[1] if K > 1 else None, b[1] if K > 1 else None, out, ws, wsb)
        return out

    check(call)


def fp8(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.float8_e4m3fn)


# few rows with few blocks per CTA, shared K, single tiles, pairs
@pytest.mark.parametrize("rows,N,K,G", [(1, 4096, 1024, 1), (16, 2048, 512, 4), (8, 4096, 4096, 4), (200, 512, 4096, 1),
                                        (160, 4096, 128, 1), (800, 4096, 512, 8), (4096, 2048, 256, 2), (2048, 4096, 2048, 1)])
def test_product(rows, N, K, G):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    A, Bw = fp8(g, rows, K), fp8(g, G * N, K)
    SA, SB = torch.rand(rows, -(-K // 128), generator=g, device="cuda"), torch.rand(G, -(-N // 128), -(-K // 128), generator=g, device="cuda")
    off = torch.from_numpy(np.linspace(0, rows, G + 1).astype(np.int32)).cuda()
    wsb = C.ec2moe_fp8_gemm_workspace_size(G, rows, N, K)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    Y = torch.empty(rows, N, device="cuda")

    def call():
        Y.fill_(3.0)
        C.ec2moe_fp8_gemm(G, rows, N, K, A, SA, off, Bw, SB, C.F32, Y, N, ws, wsb)
        return Y

    check(call)


@pytest.mark.parametrize("T,E,d,ff,act", [(2, 8, 512, 512, C.SWIGLU), (300, 4, 256, 384, C.GELU), (3000, 2, 256, 512, C.SWIGLU)])
def test_experts(T, E, d, ff, act):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    desc = C.make_desc(T=T, d=d, E=E, d_ff=ff, k=1, act=act)
    nb = lambda n: -(-n // 128)
    s = lambda *shape: torch.rand(*shape, generator=g, device="cuda") * 0.05
    w = {"W1": fp8(g, E, ff, d), "S1": s(E, nb(ff), nb(d)), "W2": fp8(g, E, d, ff), "S2": s(E, nb(d), nb(ff)), "W3": None, "S3": None}
    if act == C.SWIGLU:
        w["W3"], w["S3"] = fp8(g, E, ff, d), s(E, nb(ff), nb(d))
    X, S = fp8(g, T, d), s(T, nb(d))
    off = torch.from_numpy(np.linspace(0, T, E + 1).astype(np.int32)).cuda()
    tw = torch.ones(T, 1, device="cuda")
    perm = torch.arange(T, dtype=torch.int32, device="cuda")
    wsb = C.ec2moe_experts_fp8_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")

    def call():
        out.fill_(3.0)
        C.ec2moe_experts_fp8(desc, X, S, off, C.make_fp8_weights(**w), tw, perm, out, ws, wsb)
        return out

    check(call)
