"""The CPU oracle of the 8-bit products and the balance loss against independent
facts: enumeration of e4m3, torch's conversion, differences of the loss, and the
entry points' refusals (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C


def test_e4m3_decode_and_round_agree_on_every_value():
    v = orc.e4m3_decode(np.arange(256))
    fin = v[np.isfinite(v)]
    assert len(fin) == 254 and fin.max() == 448.0 and np.min(fin[fin > 0]) == 2.0 ** -9
    assert np.array_equal(orc.e4m3_round(fin), fin)
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, t, equal_nan=True)


def test_e4m3_round_is_nearest_even():
    fin = np.unique(np.abs(orc.e4m3_decode(np.arange(127))))
    mid = (fin[1:] + fin[:-1]) / 2
    for i, m in enumerate(mid):
        assert orc.e4m3_round(m) == fin[i if i % 2 == 0 else i + 1]  # the even mantissa
        assert orc.e4m3_round(np.nextafter(m, 0)) == fin[i]
        assert orc.e4m3_round(-np.nextafter(m, 1e9)) == -fin[i + 1]
    x = np.random.default_rng(0).normal(size=4096).astype(np.float32) * 40
    assert np.array_equal(orc.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_quantize_recovers_exact_blocks():
    """A block of e4m3 values times a power of two that holds its 448 is kept to the bit."""
    rng = np.random.default_rng(1)
    fin = orc.e4m3_decode(np.arange(127))
    x = rng.choice(fin, size=(3, 256))
    x[:, ::128] = 448.0
    x *= 2.0 ** -5
    q, s = orc.quantize(x)
    assert np.array_equal(s, np.full((3, 2), 2.0 ** -5, np.float32))
    assert np.array_equal(orc.widen(q, s), x)
    q, s = orc.quantize(np.zeros((2, 128)))
    assert not q.any() and (s > 0).all()


@pytest.mark.parametrize("K,top_groups", [(1, 0), (4, 0), (4, 2)])
def test_balance_gradient_is_the_loss_difference(K, top_groups):
    rng = np.random.default_rng(5 + K)
    T, E, k = 9, 8, 2
    O = E + (K if K > 1 else 0)
    z = rng.normal(size=(T, O))
    mask = np.array([1, 1, 0, 1, 1, 1, 0, 1])
    idx = np.argsort(-orc.gate_probabilities(z, mask, K, top_groups), 1)[:, :k]
    valid = np.ones(T, bool)
    valid[4] = False
    seg = [0, 3, 3, 9]
    args = dict(n_groups=K, coef=0.7, valid=valid, seg_offsets=seg, top_groups=top_groups)
    loss, counts, d, db = orc.balance(z, mask, idx, **args)
    assert counts.sum() == k * valid.sum() and not counts[1].any()
    # differences of a smooth function: an error of eps^2 with eps = 1e-5, and of 1e-16 / eps from rounding
    eps = 1e-5
    for t in range(T):
        for o in range(O):
            hi, lo = z.copy(), z.copy()
            hi[t, o] += eps
            lo[t, o] -= eps
            diff = (orc.balance(hi, mask, idx, **args)[0] - orc.balance(lo, mask, idx, **args)[0]) / (2 * eps)
            assert abs(diff - d[t, o]) < 1e-9, (t, o)
    assert np.allclose(db, d.sum(0), atol=1e-15)


def test_balance_of_even_loads_is_the_coefficient():
    E, T = 8, 16
    idx = (np.arange(T)[:, None] * 2 + np.arange(2)) % E
    loss, counts, d, _ = orc.balance(np.zeros((T, E)), np.ones(E), idx, 1, 0.25)
    assert abs(loss - 0.25) < 1e-15 and (counts == T * 2 // E).all() and np.abs(d).max() < 1e-17


# ----------------------------------------------------------------- refusals
A = 0x100000   # aligned placeholder address, never dereferenced
BAD = 0x100008


@pytest.fixture(scope="module")
def lib():
    B.build()
    return C.load()


def _status(fn, *args):
    try:
        fn(*args)
    except C.Ec2moeError as e:
        return e.status
    assert C.ec2moe_last_launch_count() == 0
    return C.OK


def _quant(dtype=C.BF16, n_mats=1, rows=4, cols=128, ld=128, X=A, block_rows=1, inv=None, k=0, Q=A, S=A):
    return _status(C.ec2moe_fp8_quantize, dtype, n_mats, rows, cols, ld, X, block_rows, inv, k, Q, S, 0)


def test_quantize_refusals(lib):
    assert _quant(rows=0) == C.OK and _quant(n_mats=0) == C.OK
    for bad in (dict(dtype=7), dict(rows=-1), dict(n_mats=-1), dict(cols=0), dict(ld=112), dict(block_rows=64), dict(X=None),
                dict(Q=None), dict(S=None), dict(k=2), dict(inv=A), dict(inv=A, k=1, block_rows=128),
                dict(inv=A, k=1, n_mats=2)):
        assert _quant(**bad) == C.ERR_INVALID_ARG, bad
    for bad in (dict(cols=120), dict(ld=132), dict(X=BAD), dict(Q=BAD), dict(dtype=C.F32, ld=130)):
        assert _quant(**bad) == C.ERR_MISALIGNED, bad
    for bad in (dict(inv=A, k=9), dict(rows=1 << 30, n_mats=4), dict(inv=A, k=8, rows=1 << 29),
                dict(rows=1 << 28, cols=2048, ld=2048)):
        assert _quant(**bad) == C.ERR_UNSUPPORTED, bad


def _gemm(G=1, rows=4, N=128, K=128, X=A, SA=A, off=None, W=A, SB=A, dt=C.BF16, Y=A, ldc=128, ws=A, wsb=1 << 40):
    return _status(C.ec2moe_fp8_gemm, G, rows, N, K, X, SA, off, W, SB, dt, Y, ldc, ws, wsb, 0)


def test_gemm_refusals(lib):
    assert _gemm(rows=0) == C.OK
    for bad in (dict(G=0), dict(rows=-1), dict(N=0), dict(K=0), dict(dt=3), dict(ldc=112), dict(G=2), dict(X=None),
                dict(SA=None), dict(W=None), dict(SB=None), dict(Y=None)):
        assert _gemm(**bad) == C.ERR_INVALID_ARG, bad
    for bad in (dict(N=120, ldc=120), dict(K=72), dict(ldc=132), dict(X=BAD), dict(W=BAD), dict(Y=BAD),
                dict(dt=C.F32, ldc=130)):
        assert _gemm(**bad) == C.ERR_MISALIGNED, bad
    for bad in (dict(G=129, off=A), dict(G=64, off=A, N=1 << 26, ldc=1 << 26)):
        assert _gemm(**bad) == C.ERR_UNSUPPORTED, bad
    assert C.ec2moe_fp8_gemm_workspace_size(0, 4, 128, 128) == 0


def _desc(**kw):
    base = dict(T=64, d=256, E=8, d_ff=512, k=2, n_groups=2, act=C.SWIGLU, dtype=C.BF16)
    base.update(kw)
    return C.make_desc(**base)


def _experts(desc, w=None, X=A, SX=A, off=A, tw=A, perm=A, out=A, ws=A, wsb=1 << 40):
    w = C.make_fp8_weights(W1=A, S1=A, W3=A, S3=A, W2=A, S2=A) if w is None else w
    return _status(C.ec2moe_experts_fp8, desc, X, SX, off, w, tw, perm, out, ws, wsb, 0)


def test_experts_refusals(lib):
    assert _experts(_desc(T=0)) == C.OK
    need = C.ec2moe_experts_fp8_workspace_size(_desc())
    assert need >= 64 * 2 * (512 + 4 * 4)
    assert _experts(_desc(), wsb=need - 1) == C.ERR_WORKSPACE and _experts(_desc(), ws=None) == C.ERR_WORKSPACE
    assert _experts(_desc(), ws=BAD) == C.ERR_MISALIGNED and _experts(_desc(), X=BAD) == C.ERR_MISALIGNED
    assert _experts(_desc(d_ff=520)) == C.ERR_MISALIGNED and _experts(_desc(d=264)) == C.ERR_MISALIGNED
    assert _experts(_desc(d_ff=0)) == C.ERR_INVALID_ARG and _experts(None) == C.ERR_INVALID_ARG
    for bad in (dict(SX=None), dict(off=None), dict(tw=None), dict(perm=None), dict(out=None), dict(X=None),
                dict(w=C.make_fp8_weights(W1=A, S1=A, W2=A, S2=A)), dict(w=C.make_fp8_weights(W1=A, W3=A, S3=A, W2=A, S2=A))):
        assert _experts(_desc(), **bad) == C.ERR_INVALID_ARG, bad
    assert C.ec2moe_experts_fp8_workspace_size(_desc(d_ff=520)) == 0


def test_gate_logits_refusals(lib):
    f = lambda desc, X=A, Wl=A, bl=A, Wg=A, bg=A, out=A, ws=A, wsb=1 << 40: _status(
        C.ec2moe_gate_logits, desc, X, Wl, bl, Wg, bg, out, ws, wsb, 0)
    assert f(_desc(T=0)) == C.OK
    need = C.ec2moe_gate_logits_workspace_size(_desc())
    assert f(_desc(), wsb=need - 1) == C.ERR_WORKSPACE and f(_desc(), ws=BAD) == C.ERR_MISALIGNED
    for bad in (dict(X=None), dict(Wl=None), dict(bl=None), dict(Wg=None), dict(bg=None), dict(out=None)):
        assert f(_desc(), **bad) == C.ERR_INVALID_ARG, bad
    assert f(_desc(d=260)) == C.ERR_MISALIGNED and f(_desc(), X=BAD) == C.ERR_MISALIGNED
    assert C.ec2moe_gate_logits_workspace_size(_desc(E=9)) == 0


def test_balance_refusals(lib):
    ones = np.ones(8, np.uint8)

    def f(desc=None, z=A, ld=10, mask=ones, idx=A, seg=None, n_seg=1, loss=A, counts=A, ws=A, wsb=1 << 40):
        return _status(C.ec2moe_balance_loss, _desc() if desc is None else desc, z, ld, mask, idx, None, seg, n_seg, 0.01,
                       None, loss, counts, None, None, ws, wsb, 0)

    for bad in (dict(z=None), dict(idx=None), dict(loss=None), dict(counts=None), dict(ld=9), dict(n_seg=0),
                dict(n_seg=2), dict(mask=None)):
        assert f(**bad) == C.ERR_INVALID_ARG, bad
    assert f(mask=np.zeros(8, np.uint8)) == C.ERR_ALL_MASKED
    assert f(mask=np.array([1, 0, 0, 0, 0, 0, 0, 0], np.uint8)) == C.ERR_TOO_FEW_EXPERTS
    assert f(seg=A, n_seg=1 << 29) == C.ERR_UNSUPPORTED
    need = C.ec2moe_balance_loss_workspace_size(_desc(), 1)
    assert f(wsb=need - 1) == C.ERR_WORKSPACE and f(ws=BAD) == C.ERR_MISALIGNED
    assert C.ec2moe_balance_loss_workspace_size(_desc(), 0) == 0
