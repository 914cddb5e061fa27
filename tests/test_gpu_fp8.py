"""8-bit quantiser, grouped product and experts on the GPU against the 64-bit oracle.

Tolerances, from the number formats:
* quantiser: the recipe's bits;
* product, fp32 output: the 128 exact products of a block are added in an order
  and with a truncation of the tensor core's own, at most 128 steps of 2^-23 of
  the sum of magnitudes; the scales, their product and the n_kb additions are
  further fp32 roundings.  So |error| <= tol = (128 + n_kb + 4) 2^-23 sum |a| |b|,
  element by element; a bf16 output lies between the bf16 roundings of the
  result less and plus that (rounding is monotonic);
* experts: the hidden values carry that error before they are quantised again,
  and one that lies so near a rounding boundary moves by one e4m3 step (2^-4 of
  it at most).  With K <= 1500 the error is below 1e-4 of a value of ordinary
  size, so fewer than one value in 300 moves: relative Frobenius error of at most
  2^-4 / sqrt(300) = 3.6e-3, plus 2^-9 for a bf16 output.
"""
import numpy as np
import pytest
import torch

from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests.parity import rel_fro

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
CODE = {"bf16": C.BF16, "fp32": C.F32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def quant(x, dtype, block_rows=1, n_mats=1, ld=None, inv=None, k=0, cols=None):
    """x: device [n_mats * rows, ld]."""
    cols = x.shape[1] if cols is None else cols
    rows = x.shape[0] // n_mats
    out = rows * n_mats * max(1, k)
    per = n_mats * -(-rows // 128) if block_rows == 128 else out
    Q = torch.full((out + 1, cols), 0x55, dtype=torch.uint8, device="cuda")
    S = torch.full((per + 1, -(-cols // 128)), 7.0, device="cuda")
    C.ec2moe_fp8_quantize(CODE[dtype], n_mats, rows, cols, x.shape[1] if ld is None else ld, x, block_rows, inv, k, Q, S)
    assert C.ec2moe_last_device_error() == C.OK
    assert (Q[-1] == 0x55).all() and (S[-1] == 7.0).all()  # nothing behind the rows
    return Q[:-1], S[:-1]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,ld", [(1, 16, 16), (1, 128, 128), (3, 144, 160), (65, 768, 768), (257, 1408, 1424)])
def test_rows_are_quantised_to_the_bit(dtype, rows, cols, ld):
    rng = np.random.default_rng(rows + cols)
    x = rng.normal(size=(rows, ld)).astype(np.float32) * np.exp(rng.normal(size=(rows, 1)) * 4).astype(np.float32)
    x[0, :5] = [0, -0.0, 1e-38, -3e38, 2.0 ** -140]
    if rows > 2:
        x[1] = 0
        x[2, :128] = 1e-42
    X = cuda(x, DT[dtype])
    Q, S = quant(X, dtype, cols=cols, ld=ld)
    q, s = orc.quantize(X.float().cpu().numpy()[:, :cols])
    assert np.array_equal(S.cpu().numpy(), s)
    assert np.array_equal(orc.e4m3_decode(Q.cpu().numpy()), q)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mats,rows,cols", [(1, 1, 16), (1, 128, 128), (3, 200, 272), (2, 127, 384)])
def test_weights_are_quantised_to_the_bit(dtype, mats, rows, cols):
    rng = np.random.default_rng(rows)
    X = cuda(rng.normal(size=(mats * rows, cols)).astype(np.float32) * 0.02, DT[dtype])
    Q, S = quant(X, dtype, block_rows=128, n_mats=mats)
    x = X.float().cpu().numpy()
    for m in range(mats):
        q, s = orc.quantize(x[m * rows:(m + 1) * rows], 128)
        nb = s.shape[0]
        assert np.array_equal(S.cpu().numpy()[m * nb:(m + 1) * nb], s)
        assert np.array_equal(orc.e4m3_decode(Q.cpu().numpy()[m * rows:(m + 1) * rows]), q)


@pytest.mark.parametrize("k", [1, 2, 6, 8])
def test_rows_are_placed(k):
    rng = np.random.default_rng(k)
    rows, cols = 37, 400
    X = cuda(rng.normal(size=(rows, cols)).astype(np.float32), torch.bfloat16)
    inv = rng.permutation(rows * k).astype(np.int32)
    Q, S = quant(X, "bf16", inv=cuda(inv), k=k)
    q, s = orc.quantize(X.float().cpu().numpy())
    src = np.empty(rows * k, np.int64)
    src[inv] = np.arange(rows * k) // k
    assert np.array_equal(orc.e4m3_decode(Q.cpu().numpy()), q[src]) and np.array_equal(S.cpu().numpy(), s[src])


def test_placement_outside_the_rows_is_skipped():
    X = torch.randn(4, 128, device="cuda")
    Q = torch.full((8, 128), 0x55, dtype=torch.uint8, device="cuda")
    S = torch.full((8, 1), 7.0, device="cuda")
    call = lambda inv: C.ec2moe_fp8_quantize(C.F32, 1, 4, 128, 128, X, 1, cuda(np.array(inv, np.int32)), 2, Q, S)
    call([0, 1, 2, -1, 4, 5, 6, 7])   # -1: an entry that routing skipped
    assert C.ec2moe_last_device_error() == C.OK
    call([0, 1, 2, 8, 4, 5, 6, -7])
    assert C.ec2moe_last_device_error() == C.ERR_INVALID_ARG
    assert (Q[3] == 0x55).all() and S[3, 0] == 7.0
    assert C.ec2moe_last_device_error() == C.OK


def test_nan_and_infinity():
    x = torch.randn(2, 256, device="cuda")
    x[0, 3] = float("nan")
    x[1, 200] = float("inf")
    Q, S = quant(x, "fp32")
    v = orc.e4m3_decode(Q.cpu().numpy()) * np.repeat(S.cpu().numpy(), 128, 1)
    assert np.isnan(v[0, 3]) and np.isfinite(np.delete(v[0], 3)).all()
    assert np.isfinite(v[1, :128]).all() and np.isnan(v[1, 128:]).all()


# ----------------------------------------------------------------- product
def operands(rng, rows, G, N, K, odd_scales=True):
    """e4m3 bytes and scales that no quantiser made: every finite value, scales of any size and sign."""
    a = rng.integers(0, 255, size=(rows, K), dtype=np.uint8)
    b = rng.integers(0, 255, size=(G * N, K), dtype=np.uint8)
    a[(a & 127) == 127] = 0x35
    b[(b & 127) == 127] = 0xB2
    nk, nn = -(-K // 128), -(-N // 128)
    sa = (np.exp(rng.normal(size=(rows, nk))) * 1e-3).astype(np.float32)
    sb = (np.exp(rng.normal(size=(G, nn, nk))) * rng.choice([-1, 1], size=(G, nn, nk)) * 1e-3).astype(np.float32)
    return a, sa, b, sb


def rounded(v, dtype):
    return torch.from_numpy(v).to(DT[dtype]).double().numpy() if dtype == "bf16" else v


def product_check(rng, rows, N, K, offsets, dtype, ldc=None):
    G = 1 if offsets is None else len(offsets) - 1
    a, sa, b, sb = operands(rng, rows, G, N, K)
    ldc = N if ldc is None else ldc
    Y = torch.full((rows + 1, ldc), 3.0, dtype=DT[dtype], device="cuda")
    wsb = C.ec2moe_fp8_gemm_workspace_size(G, rows, N, K)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    off = None if offsets is None else cuda(np.array(offsets, np.int32))
    C.ec2moe_fp8_gemm(G, rows, N, K, cuda(a), cuda(sa), off, cuda(b), cuda(sb), CODE[dtype], Y, ldc, ws, wsb)
    assert C.ec2moe_last_device_error() == C.OK
    y = Y.double().cpu().numpy()
    A = orc.widen(orc.e4m3_decode(a), sa)
    written = np.zeros((rows + 1, ldc), bool)
    for g in range(G):
        lo, hi = (0, rows) if offsets is None else (offsets[g], offsets[g + 1])
        W = orc.widen(orc.e4m3_decode(b[g * N:(g + 1) * N]), sb[g], 128)
        want, mag = A[lo:hi] @ W.T, np.abs(A[lo:hi]) @ np.abs(W).T
        tol = (128 + sa.shape[1] + 4) * 2.0 ** -23 * mag
        least, most = (rounded(v, dtype) for v in (want - tol, want + tol))
        assert ((least <= y[lo:hi, :N]) & (y[lo:hi, :N] <= most)).all(), (g, np.max(np.abs(y[lo:hi, :N] - want) / tol))
        written[lo:hi, :N] = True
    assert (y[~written] == 3.0).all()


SHAPES = [(1, 16, 16), (1, 256, 128), (3, 144, 272), (17, 128, 512), (64, 400, 144), (128, 256, 384), (129, 272, 256),
          (300, 528, 640), (513, 1024, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,N,K", SHAPES)
def test_dense_product(dtype, rows, N, K):
    product_check(np.random.default_rng(rows + N), rows, N, K, None, dtype, ldc=N + 16)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("counts", [[0, 1, 0, 2], [5, 0, 1, 0, 0, 3], [1] * 9, [130, 0, 7, 256, 1], [700, 30], [0, 0, 40, 0],
                                    [16, 17, 15, 33], [1] + [0] * 100 + [2, 3]])
@pytest.mark.parametrize("N,K", [(272, 400), (256, 1536)])
def test_grouped_product(dtype, counts, N, K):
    offsets = [0] + np.cumsum(counts).tolist()
    product_check(np.random.default_rng(len(counts) + N), offsets[-1], N, K, offsets, dtype)


def test_rows_of_no_group_are_left():
    product_check(np.random.default_rng(3), 50, 128, 256, [4, 9, 9, 30], "bf16")


@pytest.mark.parametrize("rows", [24, 300])
@pytest.mark.parametrize("bad", [[0, 400, 300], [0, -5, 24], [10, 2, 24]])
def test_bad_groups_are_skipped(rows, bad):
    rng = np.random.default_rng(9)
    a, sa, b, sb = operands(rng, rows, 2, 128, 256)
    Y = torch.full((rows + 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    wsb = C.ec2moe_fp8_gemm_workspace_size(2, rows, 128, 256)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    args = [cuda(v) for v in (a, sa)]
    C.ec2moe_fp8_gemm(2, rows, 128, 256, *args, cuda(np.array(bad, np.int32)), cuda(b), cuda(sb), C.BF16, Y, 128, ws, wsb)
    assert C.ec2moe_last_device_error() == C.ERR_INVALID_ARG
    assert (Y[rows:] == 3.0).all()
    assert C.ec2moe_last_device_error() == C.OK


def test_nan_stays_in_its_row():
    """A NaN row next to others of its tile, and of another group's rows in the tile, leaves them alone."""
    rng = np.random.default_rng(4)
    a, sa, b, sb = operands(rng, 20, 2, 128, 256)
    off = np.array([0, 9, 20], np.int32)
    wsb = C.ec2moe_fp8_gemm_workspace_size(2, 20, 128, 256)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")

    def call(a):
        Y = torch.empty(20, 128, device="cuda")
        C.ec2moe_fp8_gemm(2, 20, 128, 256, cuda(a), cuda(sa), cuda(off), cuda(b), cuda(sb), C.F32, Y, 128, ws, wsb)
        return Y

    want = call(a)
    a[[3, 12], 77] = 0x7F
    got = call(a)
    keep = [i for i in range(20) if i not in (3, 12)]
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[[3, 12]]).all()


# Calls of several waves of whole tiles: 256-row tiles on CTA pairs, 128-row ones on
# single CTAs; scales whose rows align to 16, 8 and 4 bytes (K = 400, 768, 272).
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,N,K,counts", [(2048, 4096, 272, None), (1000, 272, 768, None), (900, 528, 400, [512, 388]),
                                             (1040, 4096, 400, [130] * 8), (777, 2064, 768, [300, 0, 477]),
                                             (160, 4096, 16, None)])
def test_product_of_many_tiles(dtype, rows, N, K, counts):
    offsets = None if counts is None else [0] + np.cumsum(counts).tolist()
    product_check(np.random.default_rng(rows + K), rows, N, K, offsets, dtype)


# Few rows, many K blocks: a tile's sums come from several CTAs.
@pytest.mark.parametrize("rows,N,K,counts", [(1, 128, 14336, None), (100, 144, 4096, None), (3, 4096, 2048, [1, 0, 2]),
                                             (40, 1408, 2048, [0, 20, 3, 17])])
def test_product_split_over_k(rows, N, K, counts):
    offsets = None if counts is None else [0] + np.cumsum(counts).tolist()
    product_check(np.random.default_rng(rows + K), rows, N, K, offsets, "fp32")


def test_long_rows_of_offsets():
    """128 groups, most of them empty, rows at the end of a large operand."""
    counts = [0] * 128
    counts[5], counts[127] = 700, 2
    product_check(np.random.default_rng(6), 702, 128, 128, [0] + np.cumsum(counts).tolist(), "bf16")


@pytest.mark.parametrize("rows,N,K,G", [(4096, 2048, 2048, 2), (800, 4096, 2048, 8), (8, 4096, 4096, 4)],
                         ids=["pairs", "single", "few-rows"])
def test_zero_wait_budget_times_out_and_recovers(rows, N, K, G):
    rng = np.random.default_rng(rows)
    a, sa, b, sb = operands(rng, rows, G, N, K)
    dev = [cuda(v) for v in (a, sa)], [cuda(v) for v in (b, sb)]
    off = cuda(np.linspace(0, rows, G + 1).astype(np.int32))
    wsb = C.ec2moe_fp8_gemm_workspace_size(G, rows, N, K)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")

    def call():
        Y = torch.zeros(rows, N, device="cuda")
        C.ec2moe_fp8_gemm(G, rows, N, K, *dev[0], off, *dev[1], C.F32, Y, N, ws, wsb)
        return Y, C.ec2moe_last_device_error()

    ref, status = call()
    assert status == C.OK
    old = C.ec2moe_get_wait_budget()
    try:
        C.ec2moe_set_wait_budget(0)
        status = call()[1]
    finally:
        C.ec2moe_set_wait_budget(old)
    assert status == C.ERR_TIMEOUT
    again, status = call()
    assert status == C.OK and torch.equal(again, ref)


# Fewer tiles than half the SMs: the CTAs of a cluster (2 to 8) share a tile's K, in
# equal and unequal parts; rows and columns end inside the tile.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,N,K,counts", [
    (129, 4096, 4096, None), (300, 1024, 2064, None), (50, 144, 14336, None), (257, 768, 5136, None), (17, 272, 6160, None),
    (18, 16, 7184, None), (128, 5120, 3088, None), (278, 400, 2048, [200, 0, 1, 77]), (250, 528, 4112, [0, 249, 1])])
def test_product_of_clusters_that_share_k(dtype, rows, N, K, counts):
    offsets = None if counts is None else [0] + np.cumsum(counts).tolist()
    product_check(np.random.default_rng(rows + K), rows, N, K, offsets, dtype, ldc=N + 48)


def test_shared_k_gives_the_same_bits_again():
    rng = np.random.default_rng(8)
    a, sa, b, sb = (cuda(v) for v in operands(rng, 200, 1, 528, 4112))
    Y = [torch.empty(200, 528, device="cuda") for _ in range(4)]
    for y in Y:
        C.ec2moe_fp8_gemm(1, 200, 528, 4112, a, sa, None, b, sb, C.F32, y, 528, None, 0)
    assert all(torch.equal(y, Y[0]) for y in Y)


def test_shared_k_skips_bad_groups_and_times_out():
    rng = np.random.default_rng(9)
    a, sa, b, sb = (cuda(v) for v in operands(rng, 300, 2, 400, 4096))

    def call(offsets, rows=300):
        Y = torch.full((304, 400), 3.0, dtype=torch.bfloat16, device="cuda")
        C.ec2moe_fp8_gemm(2, rows, 400, 4096, a, sa, cuda(np.array(offsets, np.int32)), b, sb, C.BF16, Y, 400, None, 0)
        return Y, C.ec2moe_last_device_error()

    ref, status = call([0, 120, 300])
    assert status == C.OK
    for bad in ([0, 400, 300], [0, -5, 24], [200, 2, 300], [0, 300, 200]):
        Y, status = call(bad)
        assert status == C.ERR_INVALID_ARG and (Y[300:] == 3.0).all()
    old = C.ec2moe_get_wait_budget()
    try:
        C.ec2moe_set_wait_budget(0)
        status = call([0, 120, 300])[1]
    finally:
        C.ec2moe_set_wait_budget(old)
    assert status == C.ERR_TIMEOUT
    again, status = call([0, 120, 300])
    assert status == C.OK and torch.equal(again, ref)


# ----------------------------------------------------------------- experts
def routed(rng, T, E, k, allowed):
    idx = np.stack([rng.permutation(allowed)[:k] for _ in range(T)]).astype(np.int64)
    perm = np.argsort(idx.reshape(-1), kind="stable").astype(np.int32)
    counts = np.bincount(idx.reshape(-1), minlength=E)
    return perm, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def experts_case(rng, T, E, k, d, ff, act, allowed):
    perm, offsets = routed(rng, T, E, k, allowed)
    x = rng.normal(size=(T * k, d)).astype(np.float32)
    mk = lambda n, m: (rng.normal(size=(E * n, m)) / np.sqrt(m)).astype(np.float32)
    w = {"W1": mk(ff, d), "W3": mk(ff, d) if act == C.SWIGLU else None, "W2": mk(d, ff)}
    dev, wide = {}, {}
    for n, v in w.items():
        s = n.replace("W", "S")
        dev[n] = dev[s] = wide[n] = None
        if v is None:
            continue
        rows = v.shape[0] // E
        dev[n], dev[s] = quant(cuda(v), "fp32", block_rows=128, n_mats=E)
        q = orc.e4m3_decode(dev[n].cpu().numpy())
        sc = dev[s].cpu().numpy().reshape(E, -1, dev[s].shape[1])
        wide[n] = np.stack([orc.widen(q[e * rows:(e + 1) * rows], sc[e], 128) for e in range(E)])
    Q, S = quant(cuda(x), "fp32")
    wide["x"] = orc.widen(orc.e4m3_decode(Q.cpu().numpy()), S.cpu().numpy())
    tw = rng.uniform(0.1, 1.0, size=(T, k)).astype(np.float32)
    return perm, offsets, Q, S, dev, wide, tw


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,E,k,d,ff,act,allowed", [
    (1, 4, 2, 256, 384, C.SWIGLU, [1, 3]), (1, 1, 1, 16, 16, C.GELU, [0]), (5, 8, 2, 272, 400, C.SWIGLU, [0, 2, 3, 7]),
    (16, 4, 1, 512, 1408, C.GELU, [0, 1, 2, 3]), (70, 8, 3, 400, 528, C.GELU, list(range(8))),
    (333, 4, 2, 768, 640, C.SWIGLU, [0, 1, 3]), (1200, 3, 1, 256, 512, C.SWIGLU, [0, 1, 2]),
    (600, 1, 1, 256, 400, C.GELU, [0]), (150, 1, 1, 144, 272, C.GELU, [0]), (40, 8, 2, 272, 1408, C.SWIGLU, [2, 5])])
def test_experts(dtype, T, E, k, d, ff, act, allowed):
    rng = np.random.default_rng(T + d)
    perm, offsets, Q, S, dev, wide, tw = experts_case(rng, T, E, k, d, ff, act, allowed)
    desc = C.make_desc(T=T, d=d, E=E, d_ff=ff, k=k, act=act, dtype=CODE[dtype])
    wsb = C.ec2moe_experts_fp8_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.full((T * k + 1, d), 3.0, dtype=DT[dtype], device="cuda")
    C.ec2moe_experts_fp8(desc, Q, S, cuda(offsets), C.make_fp8_weights(**dev), cuda(tw), cuda(perm), out, ws, wsb)
    assert C.ec2moe_last_device_error() == C.OK
    assert (out[-1] == 3.0).all()
    want = orc.experts(wide["x"], offsets, wide["W1"], wide["W3"], wide["W2"], tw, perm)
    err = rel_fro(out[:-1].double().cpu().numpy(), want)
    assert err <= 3.6e-3 + (2.0 ** -9 if dtype == "bf16" else 0.0), err


# Identity weights show the hidden rows: they are the exact activation's, rounded to
# e4m3, except where that lies within GELU's and the scale's error of a tie.
@pytest.mark.parametrize("T", [8, 200, 1000])
def test_hidden_rows_are_the_exact_gelu_rounded(T):
    rng = np.random.default_rng(T)
    n = 128
    q = rng.integers(0, 255, size=(T, n), dtype=np.uint8)
    q[(q & 0x7F) == 0x7F] = 0
    s = np.exp(rng.uniform(-9, -4, size=(T, 1))).astype(np.float32)
    one, scale = cuda(np.where(np.eye(n), 0x38, 0).astype(np.uint8)), torch.ones(1, device="cuda")
    w = C.make_fp8_weights(W1=one, S1=scale, W2=one, S2=scale)
    desc = C.make_desc(T=T, d=n, E=1, d_ff=n, k=1, act=C.GELU, dtype=C.F32)
    wsb = C.ec2moe_experts_fp8_workspace_size(desc)
    out = torch.empty(T, n, device="cuda")
    off = cuda(np.array([0, T], np.int32))
    C.ec2moe_experts_fp8(desc, cuda(q), cuda(s), off, w, torch.ones(T, 1, device="cuda"),
                         torch.arange(T, dtype=torch.int32, device="cuda"), out,
                         torch.empty(wsb, dtype=torch.uint8, device="cuda"), wsb)
    assert C.ec2moe_last_device_error() == C.OK
    u = orc.e4m3_decode(q) * s.astype(np.float64)
    g = orc.gelu(u)
    to_grid = 448.0 / np.abs(g).max(axis=1, keepdims=True)
    r = g * to_grid
    codes = np.arange(256, dtype=np.uint8)
    grid = np.unique(orc.e4m3_decode(codes[(codes & 0x7F) != 0x7F]))
    at = np.clip(np.searchsorted(grid, r), 1, len(grid) - 1)
    lo, hi = grid[at - 1], grid[at]
    tie = (lo + hi) / 2
    # GELU within 1e-6 |u|, the largest value (the scale) within 1e-6 of itself
    sure = np.abs(r - tie) > 2e-6 * np.abs(u) * to_grid + 2e-6 * np.abs(r)
    want = np.where(r < tie, lo, hi)
    got = out.double().cpu().numpy() * to_grid
    assert sure.mean() > 0.99
    assert (np.abs(got - want)[sure] <= 1e-5 * np.abs(want)[sure] + 1e-12).all()


# The products back from the hidden width by clusters that share it, scattered and
# scaled by row.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,E,k,d,ff,act,allowed", [
    (100, 2, 1, 272, 2064, C.GELU, [0, 1]), (70, 4, 2, 144, 5136, C.SWIGLU, [0, 1, 3]), (150, 1, 1, 512, 3600, C.GELU, [0])])
def test_experts_share_the_hidden_width(dtype, T, E, k, d, ff, act, allowed):
    test_experts(dtype, T, E, k, d, ff, act, allowed)


@pytest.mark.parametrize("T", [6, 200])
@pytest.mark.parametrize("bad", ["offset-past-rows", "negative-offset", "decreasing-offsets", "perm-out-of-range"])
def test_experts_skip_tables_outside_the_rows(T, bad):
    rng = np.random.default_rng(T)
    E, k, d, ff = 4, 2, 128, 256
    n = T * k
    perm, offsets, Q, S, dev, _, tw = experts_case(rng, T, E, k, d, ff, C.SWIGLU, [0, 1, 2, 3])
    desc = C.make_desc(T=T, d=d, E=E, d_ff=ff, k=k, act=C.SWIGLU)
    wsb = C.ec2moe_experts_fp8_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")

    def call(offs, perm):
        out = torch.full((n + 8, d), 3.0, dtype=torch.bfloat16, device="cuda")
        C.ec2moe_experts_fp8(desc, Q, S, cuda(offs), C.make_fp8_weights(**dev), cuda(tw), cuda(perm), out, ws, wsb)
        return out, C.ec2moe_last_device_error()

    ref, status = call(offsets, perm)
    assert status == C.OK
    offs, pm = offsets.copy(), perm.copy()
    if bad == "offset-past-rows":
        offs[E] = n + 100
    elif bad == "negative-offset":
        offs[1] = -5
    elif bad == "decreasing-offsets":
        offs[2] = offs[1] - 1
    else:
        pm[3] = n + 1000
    out, status = call(offs, pm)
    assert status == C.ERR_INVALID_ARG
    assert (out[n:] == 3.0).all()
    again, status = call(offsets, perm)
    assert status == C.OK and torch.equal(again, ref)


def test_other_stream_and_repeat():
    """The same bits on a side stream, and from a call captured in a graph and replayed."""
    rng = np.random.default_rng(8)
    a, sa, b, sb = operands(rng, 40, 3, 256, 512)
    off = cuda(np.array([0, 3, 20, 40], np.int32))
    dev = [cuda(v) for v in (a, sa)], [cuda(v) for v in (b, sb)]
    wsb = C.ec2moe_fp8_gemm_workspace_size(3, 40, 256, 512)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    Y = [torch.zeros(40, 256, device="cuda") for _ in range(3)]

    def call(y, stream):
        C.ec2moe_fp8_gemm(3, 40, 256, 512, *dev[0], off, *dev[1], C.F32, y, 256, ws, wsb, stream)

    call(Y[0], None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(Y[1], side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(Y[2], None)
    graph.replay()
    assert C.ec2moe_last_device_error() == C.OK
    assert torch.equal(Y[0], Y[1]) and torch.equal(Y[0], Y[2])
