"""Waits of the bf16 layer's kernels that give up, whichever warp's it is: short budgets,
from none to microseconds, on layer calls, the standalone gate and the experts.  A call
then ends with a timeout or with its result; the next one, with the ordinary budget, gives
the ordinary bits."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from paper_2508_06024_gb300 import synth as S
from paper_2508_06024_gb300.runner import LayerRun

pytestmark = pytest.mark.gpu
BUDGETS = [0, 1, 100, 300, 1000, 3000, 10000]


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def check(call):
    """call() -> list of results."""
    ref = [t.clone() for t in call()]
    assert C.ec2moe_last_device_error() == C.OK
    old = C.ec2moe_get_wait_budget()
    for budget in BUDGETS * 2:
        try:
            C.ec2moe_set_wait_budget(budget)
            got = [t.clone() for t in call()]
            status = C.ec2moe_last_device_error()
        finally:
            C.ec2moe_set_wait_budget(old)
        # a timeout, or what skips tables that a kernel before gave up on
        assert status in (C.OK, C.ERR_TIMEOUT)
        if status == C.OK:
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
        got = call()
        assert C.ec2moe_last_device_error() == C.OK
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


LAYERS = [S.preset("switch_bf16", T=512, seed=31), S.preset("switch_bf16", T=100, d_ff=256, seed=35),
          S.preset("finegrained_bf16", T=300, seed=32), S.preset("finegrained_bf16", T=3000, d_ff=256, seed=36),
          S.preset("mixtral_bf16", T=2048, E=4, n_allowed=3, d_ff=1024, seed=33),
          S.preset("decode_bf16", T=1, d_ff=2048, seed=34), S.preset("decode_bf16", T=40, d_ff=1024, seed=37)]


@pytest.mark.parametrize("cfg", LAYERS, ids=["switch", "short-k", "finegrained", "finegrained-long", "pairs", "one-token", "decode"])
def test_layer(cfg):
    run = LayerRun(cfg, S.make_inputs(cfg, device="cuda"))

    def call():
        return [run.forward()]

    check(call)


# clusters that share d_model, single tiles, prepared gate rows
@pytest.mark.parametrize("T,d,E,K,k", [(100, 512, 16, 4, 2), (700, 4096, 8, 2, 2), (5000, 768, 16, 1, 1), (20000, 2048, 64, 8, 6)])
def test_gate(T, d, E, K, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    X = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    W = [torch.randn(n, d, generator=g, device="cuda") / d ** 0.5 for n in (E, K)]
    b = [torch.randn(n, generator=g, device="cuda") for n in (E, K)]
    desc = C.make_desc(T=T, d=d, E=E, d_ff=0, k=k, n_groups=K)
    mask = C.host_mask(torch.ones(E, dtype=torch.uint8))
    idx = torch.empty(T, k, dtype=torch.int32, device="cuda")
    w = torch.empty(T, k, device="cuda")

    def call():
        C.ec2moe_gate(desc, X, W[0], b[0], W[1] if K > 1 else None, b[1] if K > 1 else None, mask, idx, w)
        return [idx, w]

    check(call)


# tokens on the MMA's N side; single tiles; few rows
@pytest.mark.parametrize("rows,d,ff,act", [([200, 300, 250, 274], 2592, 2464, C.SWIGLU), ([129, 5, 0, 300], 256, 512, C.GELU),
                                           ([3, 0, 7, 1], 512, 1024, C.SWIGLU)])
def test_experts(rows, d, ff, act):
    g = torch.Generator(device="cuda")
    g.manual_seed(ff)
    E, n = len(rows), sum(rows)
    t = lambda *s: (torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5).to(torch.bfloat16)
    X, W1, W3, W2 = t(n, d), t(E, ff, d), t(E, ff, d), t(E, d, ff)
    off = torch.tensor([sum(rows[:i]) for i in range(E + 1)], dtype=torch.int32, device="cuda")
    desc = C.make_desc(T=n, d=d, E=E, d_ff=ff, k=1, act=act)
    wsb = C.ec2moe_experts_workspace_size(desc)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    perm = torch.randperm(n, generator=g, device="cuda").int()
    w = torch.rand(n, generator=g, device="cuda")
    out = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")

    def call():
        out.fill_(3.0)
        C.ec2moe_experts(desc, X, off, W1, W3 if act == C.SWIGLU else None, W2, w, perm, out, ws, wsb)
        return [out]

    check(call)
