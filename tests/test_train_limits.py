"""Refusals of the norm, the activation and the grouped products: host checks, before anything reaches a GPU."""
import math

import pytest

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

A = 0x100000   # aligned addresses that are never reached
BAD = 0x100008


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def status(fn, **kw):
    try:
        fn(**kw)
    except C.Ec2moeError as e:
        return e.status
    return C.OK


NORM = dict(dtype=C.BF16, y_dtype=C.BF16, rows=4, cols=64, ld=64, X=A, residual=A, weight=A, eps=1e-5, H=A, rstd=A, Y=A,
            Q=A, scale=A, stream=0)
BACK = dict(dtype=C.BF16, y_dtype=C.BF16, rows=4, cols=64, ld=64, dY=A, H=A, rstd=A, weight=A, dH=A, dX=A, d_weight=A,
            workspace=A, ws_bytes=1 << 30, stream=0)
ACT = dict(dtype=C.BF16, act=C.SWIGLU, rows=4, cols=64, ld=128, U=A, V=A, perm=A, row_scale=A, H=A, stream=0)
ACT_BACK = dict(ACT, dH=A, dU=A, dV=A, d_row_scale=A)
FWD = dict(n_groups=2, rows=4, N=64, K=32, A=A, lda=32, offsets=A, B=A, perm=A, out_dtype=C.BF16, out=A, ldc=64, workspace=A,
           ws_bytes=1 << 40, stream=0)
DGRAD = dict(n_groups=2, rows=4, N=64, K=32, dC=A, lddc=64, offsets=A, B=A, perm=A, out_dtype=C.BF16, dA=A, ldda=32,
             workspace=A, ws_bytes=1 << 40, stream=0)
WGRAD = dict(n_groups=2, rows=4, N=64, K=32, dC=A, lddc=64, A=A, lda=32, offsets=A, out_dtype=C.F32, accumulate=0, dB=A,
             workspace=A, ws_bytes=1 << 40, stream=0)
INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = C.ERR_INVALID_ARG, C.ERR_UNSUPPORTED, C.ERR_MISALIGNED, C.ERR_WORKSPACE

CASES = [
    (C.ec2moe_rmsnorm, NORM, [
        (dict(dtype=2), INVALID), (dict(y_dtype=7), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID),
        (dict(ld=56), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID),
        (dict(Q=None), INVALID), (dict(scale=None), INVALID), (dict(H=None, rstd=None, Y=None, Q=None, scale=None), INVALID),
        (dict(X=None), INVALID), (dict(cols=60), MISALIGNED), (dict(ld=68), MISALIGNED), (dict(cols=56, ld=56), MISALIGNED),
        (dict(cols=16392, ld=16392, Q=None, scale=None), UNSUPPORTED), (dict(X=BAD), MISALIGNED), (dict(residual=BAD), MISALIGNED),
        (dict(weight=BAD), MISALIGNED), (dict(H=BAD), MISALIGNED), (dict(Y=BAD), MISALIGNED), (dict(Q=BAD), MISALIGNED),
        (dict(rows=0, X=None), C.OK)]),
    (C.ec2moe_rmsnorm_backward, BACK, [
        (dict(dtype=2), INVALID), (dict(y_dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(ld=56), INVALID),
        (dict(dY=None), INVALID), (dict(H=None), INVALID), (dict(rstd=None), INVALID), (dict(dX=None), INVALID),
        (dict(cols=60), MISALIGNED), (dict(ld=68), MISALIGNED), (dict(cols=16392, ld=16392), UNSUPPORTED),
        (dict(dY=BAD), MISALIGNED), (dict(dH=BAD), MISALIGNED), (dict(weight=BAD), MISALIGNED), (dict(d_weight=BAD), MISALIGNED),
        (dict(workspace=BAD), MISALIGNED), (dict(workspace=None), WORKSPACE), (dict(accumulate=2), INVALID), (dict(rows=0, d_weight=None), C.OK)]),
    (C.ec2moe_activation, ACT, [
        (dict(dtype=2), INVALID), (dict(act=2), INVALID), (dict(rows=-1), INVALID), (dict(ld=56), INVALID), (dict(U=None), INVALID),
        (dict(V=None), INVALID), (dict(H=None), INVALID), (dict(cols=60), MISALIGNED), (dict(ld=132), MISALIGNED),
        (dict(U=BAD), MISALIGNED), (dict(V=BAD), MISALIGNED), (dict(H=BAD), MISALIGNED), (dict(rows=0, U=None), C.OK)]),
    (C.ec2moe_activation_backward, ACT_BACK, [
        (dict(dtype=2), INVALID), (dict(act=-1), INVALID), (dict(rows=-1), INVALID), (dict(ld=56), INVALID), (dict(U=None), INVALID),
        (dict(dH=None), INVALID), (dict(dU=None), INVALID), (dict(dV=None), INVALID), (dict(cols=60), MISALIGNED),
        (dict(dV=BAD), MISALIGNED), (dict(dU=BAD), MISALIGNED), (dict(dH=BAD), MISALIGNED), (dict(H=BAD), MISALIGNED),
        (dict(rows=0, U=None), C.OK)]),
    (C.ec2moe_grouped_gemm, FWD, [
        (dict(n_groups=0), INVALID), (dict(rows=-1), INVALID), (dict(N=0), INVALID), (dict(K=-8), INVALID), (dict(lda=24), INVALID),
        (dict(ldc=56), INVALID), (dict(out_dtype=3), INVALID), (dict(offsets=None), INVALID), (dict(A=None), INVALID),
        (dict(B=None), INVALID), (dict(out=None), INVALID), (dict(n_groups=129), UNSUPPORTED), (dict(N=60), MISALIGNED),
        (dict(K=28), MISALIGNED), (dict(lda=36), MISALIGNED), (dict(ldc=68), MISALIGNED), (dict(A=BAD), MISALIGNED),
        (dict(B=BAD), MISALIGNED), (dict(out=BAD), MISALIGNED), (dict(rows=2 ** 31 - 1), UNSUPPORTED),
        (dict(N=2 ** 31 - 8, ldc=2 ** 31 - 8), UNSUPPORTED), (dict(rows=0, A=None), C.OK)]),
    (C.ec2moe_grouped_gemm_dgrad, DGRAD, [
        (dict(n_groups=0), INVALID), (dict(lddc=56), INVALID), (dict(ldda=24), INVALID), (dict(offsets=None), INVALID),
        (dict(dC=None), INVALID), (dict(B=None), INVALID), (dict(dA=None), INVALID), (dict(N=60), MISALIGNED),
        (dict(lddc=68), MISALIGNED), (dict(ldda=36), MISALIGNED), (dict(dC=BAD), MISALIGNED), (dict(dA=BAD), MISALIGNED),
        (dict(n_groups=200), UNSUPPORTED), (dict(rows=0, dC=None), C.OK)]),
    (C.ec2moe_grouped_gemm_wgrad, WGRAD, [
        (dict(n_groups=0), INVALID), (dict(lddc=56), INVALID), (dict(lda=24), INVALID), (dict(offsets=None), INVALID),
        (dict(accumulate=2), INVALID), (dict(accumulate=1, out_dtype=C.BF16), INVALID), (dict(dC=None), INVALID),
        (dict(A=None), INVALID), (dict(dB=None), INVALID), (dict(dB=BAD), MISALIGNED), (dict(A=BAD), MISALIGNED),
        (dict(lda=36), MISALIGNED), (dict(lddc=68), MISALIGNED), (dict(N=2 ** 20, K=2 ** 20, lddc=2 ** 20, lda=2 ** 20), UNSUPPORTED),
        (dict(rows=0, accumulate=1), C.OK)]),
]


@pytest.mark.parametrize("fn,base,change,want", [(f, b, c, w) for f, b, cases in CASES for c, w in cases],
                         ids=lambda v: getattr(v, "__name__", None) or (str(v)[:60] if isinstance(v, dict) and len(v) < 6 else ""))
def test_refusals(fn, base, change, want):
    assert status(fn, **{**base, **change}) == want


def test_workspace_sizes():
    assert C.ec2moe_rmsnorm_backward_workspace_size(0, 64) == 0
    assert C.ec2moe_rmsnorm_backward_workspace_size(4, 60) == 0
    assert C.ec2moe_rmsnorm_backward_workspace_size(4, 16392) == 0
    assert C.ec2moe_grouped_gemm_workspace_size(2, 4, 60, 32) == 0
    assert C.ec2moe_grouped_gemm_workspace_size(2, 0, 64, 32) == 0
