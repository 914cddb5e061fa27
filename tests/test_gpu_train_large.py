"""Element offsets beyond 32 bits: the last rows of operands and results of more than 2^31 elements
are what a call on those rows alone gives, bit by bit (each row, and each group, is computed for itself)."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
LAST = 200


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()
    yield
    torch.cuda.empty_cache()


def long(rows, cols, last):
    """Zeros [rows, cols] whose last rows are `last`."""
    t = torch.zeros(rows, cols, dtype=last.dtype, device="cuda")
    t[rows - last.shape[0]:] = last
    return t


def rand(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(BF)


def test_norm():
    rows, cols = 140000, 16384
    x, w = rand(LAST, cols), 1 + 0.1 * torch.randn(cols, device="cuda")
    out = {}
    for n in (rows, LAST):
        X = long(n, cols, x)
        Y, rstd = torch.empty_like(X), torch.empty(n, device="cuda")
        Q, S = torch.empty(n, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(n, cols // 128, device="cuda")
        C.ec2moe_rmsnorm(C.BF16, C.BF16, n, cols, cols, X, None, w, 1e-5, None, rstd, Y, Q, S)
        ws = torch.empty(C.ec2moe_rmsnorm_backward_workspace_size(n, cols), dtype=torch.uint8, device="cuda")
        # the gradient, in the place of its operand
        C.ec2moe_rmsnorm_backward(C.BF16, C.BF16, n, cols, cols, Y, X, rstd, w, None, X, None, ws, ws.numel())
        assert C.ec2moe_last_device_error() == C.OK
        out[n] = [t[n - LAST:].clone() for t in (Y, rstd, Q.view(torch.uint8), S, X)]
        del X, Y, Q, S
    assert all(torch.equal(a, b) for a, b in zip(out[rows], out[LAST]))


def test_activation():
    rows, cols = 160000, 14336
    u, dh = rand(LAST, cols), rand(LAST, cols, seed=1)
    out = {}
    for n in (rows, LAST):
        U, dH = long(n, cols, u), long(n, cols, dh)
        H = torch.empty_like(U)
        C.ec2moe_activation(C.BF16, C.GELU, n, cols, cols, U, None, None, None, H)
        C.ec2moe_activation_backward(C.BF16, C.GELU, n, cols, cols, U, None, None, None, dH, U, None, dH, None)
        out[n] = [t[n - LAST:].clone() for t in (H, U, dH)]
        del U, dH, H
    assert all(torch.equal(a, b) for a, b in zip(out[rows], out[LAST]))


@pytest.mark.parametrize("form", ["fwd", "dgrad"])
@pytest.mark.parametrize("wide", ["operand", "result"])
def test_rows_of_products(form, wide):
    """`rows` x 14336 elements of the operand, or of the result; the last group's rows, to other rows through perm."""
    rows, deep, cols = 160000, *((14336, 64) if wide == "operand" else (64, 14336))
    x = rand(LAST, deep)
    W = rand(2, *((cols, deep) if form == "fwd" else (deep, cols)), seed=1)
    N, K = W.shape[1:]
    fn = C.ec2moe_grouped_gemm if form == "fwd" else C.ec2moe_grouped_gemm_dgrad
    out = {}
    for n in (rows, LAST):
        X = long(n, deep, x)
        Y = torch.empty(n, cols, dtype=BF, device="cuda")
        offsets = torch.tensor([0, n - LAST, n], dtype=torch.int32, device="cuda")
        perm = torch.arange(n, dtype=torch.int32, device="cuda")
        perm[n - LAST:] = perm[n - LAST:].flip(0)
        ws = torch.empty(max(16, C.ec2moe_grouped_gemm_workspace_size(2, n, N, K)), dtype=torch.uint8, device="cuda")
        fn(2, n, N, K, X, deep, offsets, W, perm, C.BF16, Y, cols, ws, ws.numel())
        assert C.ec2moe_last_device_error() == C.OK
        out[n] = Y[n - LAST:].double()
        del X, Y, ws
    want = (x.double() @ (W[1].double().T if form == "fwd" else W[1].double())).flip(0)
    # sums may be cut into ranges in one of the two calls; of at most 896 steps each cuts 2^-23 of a sum of some 400
    for got in out.values():
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3 * deep ** 0.5).all())


def test_weights_of_a_product():
    G, N, K, rows = 40, 8192, 8192, 80
    X, A = rand(rows, N), rand(rows, K, seed=1)
    offsets = torch.arange(0, rows + 1, 2, dtype=torch.int32, device="cuda")
    dB = torch.full((G, N, K), 3.0, dtype=BF, device="cuda")
    ws = torch.empty(max(16, C.ec2moe_grouped_gemm_workspace_size(G, rows, N, K)), dtype=torch.uint8, device="cuda")
    C.ec2moe_grouped_gemm_wgrad(G, rows, N, K, X, N, A, K, offsets, C.BF16, 0, dB, ws, ws.numel())
    assert C.ec2moe_last_device_error() == C.OK
    for g in (0, 31, 32, G - 1):
        want = X[2 * g:2 * g + 2].double().T @ A[2 * g:2 * g + 2].double()
        assert bool(((dB[g].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all())
