"""Group tables that go back and forth: groups own no row twice, so that nothing is
written behind the workspace, whose size counts every row once."""
import numpy as np
import pytest
import torch

from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu
GUARD = 8 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def guarded(n):
    """A workspace of n bytes inside a larger allocation whose rest is filled."""
    n = max(16, n)
    return torch.full((n + GUARD,), 0x5A, dtype=torch.uint8, device="cuda"), n


def fp8(rng, *shape):
    q = rng.integers(0, 255, size=shape, dtype=np.uint8)
    q[(q & 127) == 127] = 0x35
    return q


def owned(offsets, rows):
    """The rows [lo, hi) of each group by the stated rule."""
    reach, out = 0, []
    for a, b in zip(offsets, offsets[1:]):
        ok = 0 <= a < b <= rows and a >= reach
        out.append((a, b) if ok else (0, 0))
        if 0 <= a < b <= rows:
            reach = max(reach, b)
    return out


# few rows (partial sums in the workspace), clusters that share K, whole tiles, pairs
@pytest.mark.parametrize("rows,N,K,G", [(128, 4096, 512, 8), (40, 256, 1536, 40), (300, 272, 2048, 8), (1200, 2048, 256, 8),
                                        (8192, 2048, 128, 4)])
@pytest.mark.parametrize("table", ["back-and-forth", "halves", "nested"])
def test_groups_own_no_row_twice(rows, N, K, G, table):
    rng = np.random.default_rng(rows + G)
    half = rows // 2
    offsets = {"back-and-forth": [0, rows] * G, "halves": [0, half, 0, rows, half - 1, rows] * G,
               "nested": [half, rows, 1, rows - 1, rows, 2, 5] * G}[table][:G + 1]
    a, b = fp8(rng, rows, K), fp8(rng, G * N, K)
    sa = np.exp(rng.normal(size=(rows, -(-K // 128)))).astype(np.float32) * 1e-3
    sb = np.exp(rng.normal(size=(G, -(-N // 128), -(-K // 128)))).astype(np.float32) * 1e-3
    ws, n = guarded(C.ec2moe_fp8_gemm_workspace_size(G, rows, N, K))
    dev = [cuda(v) for v in (a, sa, b, sb)]

    def call(offs):
        Y = torch.full((rows + 1, N), 3.0, device="cuda")
        C.ec2moe_fp8_gemm(G, rows, N, K, dev[0], dev[1], cuda(np.array(offs, np.int32)), dev[2], dev[3], C.F32, Y, N, ws, n)
        return Y, C.ec2moe_last_device_error()

    Y, status = call(offsets)
    assert status == C.ERR_INVALID_ARG
    assert (ws[n:] == 0x5A).all()
    want = torch.full_like(Y, 3.0)
    for g, (lo, hi) in enumerate(owned(offsets, rows)):
        if hi > lo:
            # the same rows by themselves; sums of few rows may be cut elsewhere
            A = orc.widen(orc.e4m3_decode(a[lo:hi]), sa[lo:hi])
            W = orc.widen(orc.e4m3_decode(b[g * N:(g + 1) * N]), sb[g], 128)
            want[lo:hi] = cuda((A @ W.T).astype(np.float32))
            tol = (128 + K / 128 + 5) * 2.0 ** -23 * cuda(np.abs(A) @ np.abs(W).T)
            assert ((Y[lo:hi].double() - want[lo:hi].double()).abs() <= tol).all()
            Y[lo:hi] = want[lo:hi]
    assert torch.equal(Y, want)  # rows of no group are left
    good = np.linspace(0, rows, G + 1).astype(int).tolist()
    assert call(good)[1] == C.OK and (ws[n:] == 0x5A).all()


@pytest.mark.parametrize("T,d,ff", [(64, 512, 256), (600, 256, 384)])
@pytest.mark.parametrize("act", [C.GELU, C.SWIGLU])
def test_experts_own_no_row_twice(T, d, ff, act):
    rng = np.random.default_rng(T)
    E, k = 8, 2
    n = T * k
    desc = C.make_desc(T=T, d=d, E=E, d_ff=ff, k=k, act=act)
    ones = lambda *s: torch.full(s, 1e-3, device="cuda")
    w = {"W1": cuda(fp8(rng, E, ff, d)), "S1": ones(E, -(-ff // 128), -(-d // 128)), "W2": cuda(fp8(rng, E, d, ff)),
         "S2": ones(E, -(-d // 128), -(-ff // 128)), "W3": None, "S3": None}
    if act == C.SWIGLU:
        w["W3"], w["S3"] = cuda(fp8(rng, E, ff, d)), w["S1"]
    X, S = cuda(fp8(rng, n, d)), ones(n, -(-d // 128))
    ws, size = guarded(C.ec2moe_experts_fp8_workspace_size(desc))
    tw = torch.ones(T, k, device="cuda")
    perm = torch.arange(n, dtype=torch.int32, device="cuda")

    def call(offsets):
        out = torch.full((n + 1, d), 3.0, dtype=torch.bfloat16, device="cuda")
        C.ec2moe_experts_fp8(desc, X, S, cuda(np.array(offsets, np.int32)), C.make_fp8_weights(**w), tw, perm, out, ws, size)
        return out, C.ec2moe_last_device_error()

    out, status = call([0, n] * (E // 2) + [0])
    assert status == C.ERR_INVALID_ARG and (ws[size:] == 0x5A).all() and (out[n] == 3.0).all()
    first, status = call([0] + [n] * E)  # all rows the first expert's
    assert status == C.OK and (ws[size:] == 0x5A).all()
    assert torch.equal(out, first)
