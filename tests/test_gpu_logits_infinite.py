"""Gate logits of activations and gate rows with infinities, NaN and weights beyond
bf16's range: what the definition gives in 64 bits, and no other token's or gate row's
logits change by a bit."""
import numpy as np
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def logits(X, W, b, E, K):
    T, d = X.shape
    desc = C.make_desc(T=T, d=d, E=E, d_ff=0, k=1, n_groups=K, dtype=C.BF16 if X.dtype == torch.bfloat16 else C.F32)
    wsb = C.ec2moe_gate_logits_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.full((T + 1, W.shape[0]), 7.0, device="cuda")
    two = [W[:E].clone(), b[:E].clone(), W[E:].clone(), b[E:].clone()]
    C.ec2moe_gate_logits(desc, X, two[0], two[1], two[2] if K > 1 else None, two[3] if K > 1 else None, out, ws, wsb)
    assert C.ec2moe_last_device_error() == C.OK and (out[-1] == 7.0).all()
    return out[:-1]


# clusters, single tiles, more than 128 gate rows
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E,K", [(1, 8, 1, 1), (5, 264, 10, 5), (200, 512, 16, 4), (20000, 136, 16, 4), (300, 520, 128, 16)])
def test_infinities(dtype, T, d, E, K):
    rng = np.random.default_rng(T)
    O = E + (K if K > 1 else 0)
    X = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).cuda().to(dtype)
    W = torch.from_numpy((rng.normal(size=(O, d)) / np.sqrt(d)).astype(np.float32)).cuda()
    b = torch.from_numpy(rng.normal(size=O).astype(np.float32)).cuda()
    before = logits(X, W, b, E, K)
    inf = float("inf")
    rows, cols = [], []

    def put(t, *values):
        t = t % T
        for c, v in values:
            X[t, c] = v
        rows.append(t)

    put(0, (5, inf))
    if T > 4:
        put(3, (7, -inf))
        put(T - 1, (0, inf))
        put(T // 2, (1, inf), (2, -inf))
        put(2, (d - 1, float("nan")))
        W[0, 5] = 0.0  # against an infinity: NaN
        W[O - 1, 0] = inf
        W[O // 2, 3] = 3.4e38  # beyond bf16's largest
        cols += [0, O - 1, O // 2]
    got = logits(X, W, b, E, K)
    want = torch.from_numpy((X.double().cpu().numpy() @ W.double().cpu().numpy().T) + b.double().cpu().numpy()).cuda().float()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()], want[want.isinf()])
    keep = torch.ones(T, O, dtype=torch.bool, device="cuda")
    keep[rows] = False
    keep[:, cols] = False
    assert torch.equal(got[keep], before[keep])
    # 3.4e38 x_3 is most of its sum: the rest is below fp32's last bit of it
    fin = got.isfinite() & ~keep
    mag = X.double().abs() @ W.double().abs().T + b.double().abs()
    ok = fin & mag.isfinite()
    assert ((got.double() - want.double()).abs()[ok] <= (32 + d / 512 + 9) * 2.0 ** -23 * mag[ok]).all()
