"""The norm with the residual's addition, its 8-bit rows and its gradient, against 64 bits.

Errors, relative: the sum of the squares at most (cols / 8 threads add in order and then in a
tree, so at most 4 x 8 + 10 additions in a thread's chain) 48 2^-24; rstd half of that and
three roundings, y and the gradients' elementwise steps a few roundings of 2^-24 more: 64
2^-24 covers them.  bf16 results are rounded by 2^-8.  e4m3 values agree where the fp32 value is
not within its error of a tie; there they differ by one step, 2^-3 relative.
"""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests import train_reference as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
CODE = {BF: C.BF16, F32: C.F32}
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
E = 64 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def rand(*shape, dtype=F32, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(shape[0], shape[1] + pad, generator=g, device="cuda").to(dtype) if len(shape) == 2 else \
        torch.randn(*shape, generator=g, device="cuda").to(dtype)
    return t[:, :shape[1]] if len(shape) == 2 else t


def near(got, want, dtype, scale=None):
    """|got - want| within E of `scale` (default: of itself) and the type's rounding."""
    want = want.double()
    scale = want.abs() if scale is None else scale
    err = (got.double() - want).abs()
    bound = HALF[dtype] * want.abs() + E * scale + 1e-37
    assert bool((err <= bound).all()), float((err / bound).max())


SHAPES = [(1, 8), (3, 16), (5, 24), (1, 4096), (257, 768), (64, 2048), (700, 4096), (33, 5008), (9, 16384), (311, 9000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,y_dtype", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("residual", [True, False])
def test_forward(rows, cols, dtype, y_dtype, residual):
    pad = 8
    x, r = rand(rows, cols, dtype=dtype, pad=pad), rand(rows, cols, dtype=dtype, seed=1, pad=pad) if residual else None
    w = 1 + 0.3 * rand(cols, seed=2)
    q8 = cols % 16 == 0
    H, rstd = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(rows, device="cuda")
    Y = torch.empty(rows, cols, dtype=y_dtype, device="cuda")
    Q = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda") if q8 else None
    S = torch.empty(rows, -(-cols // 128), device="cuda") if q8 else None
    C.ec2moe_rmsnorm(CODE[dtype], CODE[y_dtype], rows, cols, cols + pad, x, r, w, 1e-5, H, rstd, Y, Q, S)
    h, rs, y = ref.rmsnorm(x, r, w, 1e-5)
    near(H, h, dtype)
    near(rstd, rs, F32)
    near(Y, y, y_dtype)
    if not q8:
        return
    blocks = torch.nn.functional.pad(y, (0, -cols % 128)).view(rows, -1, 128)
    s = blocks.abs().amax(2).clamp_min(2.0 ** -96) / 448
    near(S, s, F32)
    want = (ref.to_e4m3(blocks / s[:, :, None])).view(rows, -1)[:, :cols]
    got = Q.to(F32).double()
    # one step (2^-3 relative, 2^-9 below the normal range) where the value is next to a tie
    assert bool(((got - want).abs() <= 2.0 ** -3 * want.abs().clamp_min(2.0 ** -6)).all())
    assert float((got != want).double().mean()) <= max(1e-3, 2.0 / got.numel())


def test_selected_outputs_and_aliases():
    rows, cols = 130, 2048
    x, r, w = rand(rows, cols, dtype=BF), rand(rows, cols, dtype=BF, seed=1), 1 + 0.3 * rand(cols, seed=2)
    Y = torch.empty(rows, cols, dtype=BF, device="cuda")
    H = torch.empty_like(Y)
    C.ec2moe_rmsnorm(C.BF16, C.BF16, rows, cols, cols, x, r, w, 1e-5, H, None, Y)
    for alias in ("residual", "x"):
        a, b = x.clone(), r.clone()
        into = b if alias == "residual" else a
        Y2 = torch.empty_like(Y)
        C.ec2moe_rmsnorm(C.BF16, C.BF16, rows, cols, cols, a, b, w, 1e-5, into, None, Y2)
        assert torch.equal(into, H) and torch.equal(Y2, Y)
    only = torch.empty(rows, device="cuda")
    C.ec2moe_rmsnorm(C.BF16, C.BF16, rows, cols, cols, x, r, None, 1e-5, None, only)
    near(only, ref.rmsnorm(x, r, None, 1e-5)[1], F32)
    Q, S = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, cols // 128, device="cuda")
    C.ec2moe_rmsnorm(C.BF16, C.F32, rows, cols, cols, x, r, w, 1e-5, None, None, None, Q, S)
    # the quantiser's own rows, from the y that is rounded to fp32
    Yf = torch.empty(rows, cols, device="cuda")
    C.ec2moe_rmsnorm(C.BF16, C.F32, rows, cols, cols, x, r, w, 1e-5, None, None, Yf)
    Q2, S2 = torch.empty_like(Q), torch.empty_like(S)
    C.ec2moe_fp8_quantize(C.F32, 1, rows, cols, cols, Yf, 1, None, 0, Q2, S2)
    # to the next value where one of the two is beside a tie; the scales to an fp32 rounding
    a, b = Q.to(F32), Q2.to(F32)
    assert bool(((a - b).abs() <= 2.0 ** -3 * torch.maximum(a.abs(), b.abs())).all()) and float((a != b).float().mean()) < 1e-4
    near(S, S2, F32)


def test_unusual_values():
    cols = 256
    x = rand(6, cols, dtype=F32)
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 7] = float("nan")
    x[3] *= 1e-25
    x[4] *= 1e15
    Y, rstd = torch.empty(6, cols, device="cuda"), torch.empty(6, device="cuda")
    Q, S = torch.empty(6, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, 2, device="cuda")
    C.ec2moe_rmsnorm(C.F32, C.F32, 6, cols, cols, x, None, None, 1e-6, None, rstd, Y, Q, S)
    _, _, y = ref.rmsnorm(x, None, None, 1e-6)
    assert bool((Y[0] == 0).all()) and bool((Q[0].to(F32) == 0).all()) and bool((S[0] == 2.0 ** -96 / 448).all())
    assert bool(torch.isnan(Y[1, 5])) and bool((Y[1, :5] == 0).all()) and float(rstd[1]) == 0
    assert bool(torch.isnan(Y[2]).all())
    near(Y[3:], y[3:], F32)


@pytest.mark.parametrize("rows,cols", SHAPES + [(4001, 512)])
@pytest.mark.parametrize("dtype,y_dtype", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("with_dh", [True, False])
def test_backward(rows, cols, dtype, y_dtype, with_dh):
    h, dh = rand(rows, cols, dtype=dtype), rand(rows, cols, dtype=dtype, seed=1) if with_dh else None
    dy, w = rand(rows, cols, dtype=y_dtype, seed=2, pad=8), 1 + 0.3 * rand(cols, seed=3)
    rstd = ref.rmsnorm(h, None, None, 1e-5)[1].float()
    dx, dw = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(max(16, C.ec2moe_rmsnorm_backward_workspace_size(rows, cols)), dtype=torch.uint8, device="cuda")

    def call(dH, dX, dW):
        C.ec2moe_rmsnorm_backward(CODE[dtype], CODE[y_dtype], rows, cols, cols + 8, dy, h, rstd, w, dH, dX, dW, ws, ws.numel())

    call(dh, dx, dw)
    want, dw_want = ref.rmsnorm_backward(dy, h, rstd, w, dh)
    g, xhat = dy.double() * w.double(), h.double() * rstd.double()[:, None]
    scale = rstd.double()[:, None] * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    scale = scale if dh is None else scale + dh.double().abs()
    near(dx, want, dtype, scale)
    # a column's sum: a chain of at most rows additions in fp32
    terms = (dy.double() * xhat).abs().sum(0)
    assert bool(((dw.double() - dw_want).abs() <= (rows + 16) * 2.0 ** -24 * terms + 1e-30).all())
    again, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    call(dh, again, dw2)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)
    C.ec2moe_rmsnorm_backward(CODE[dtype], CODE[y_dtype], rows, cols, cols + 8, dy, h, rstd, w, dh, again, dw2, ws, ws.numel(),
                              accumulate=1)
    assert torch.equal(dw2, dw + dw)
    again.zero_()
    call(dh, again, None)
    assert torch.equal(again, dx)
    if with_dh:
        call(dh, dh, dw2)  # in the gradient's own place
        assert torch.equal(dh, dx) and torch.equal(dw2, dw)


def test_backward_against_differences():
    """dX and d_weight against central differences of the 64-bit forward, fp32 operands."""
    rows, cols, eps = 2, 24, 1e-3
    x, w = rand(rows, cols), 1 + 0.3 * rand(cols, seed=1)
    dy = rand(rows, cols, seed=2)
    Y, rstd = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda")
    C.ec2moe_rmsnorm(C.F32, C.F32, rows, cols, cols, x, None, w, eps, None, rstd, Y)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(C.ec2moe_rmsnorm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    C.ec2moe_rmsnorm_backward(C.F32, C.F32, rows, cols, cols, dy, x, rstd, w, None, dx, dw, ws, ws.numel())
    e = 1e-4

    def loss(x_, w_):
        return float((ref.rmsnorm(x_, None, w_, eps)[2] * dy.double()).sum())

    for r in range(rows):
        for c in range(cols):
            step = torch.zeros_like(x, dtype=torch.float64)
            step[r, c] = e
            diff = (loss(x.double() + step, w.double()) - loss(x.double() - step, w.double())) / (2 * e)
            assert abs(diff - float(dx[r, c])) < 1e-4  # e^2 times the third derivative, and fp32
    for c in range(cols):
        step = torch.zeros(cols, dtype=torch.float64, device="cuda")
        step[c] = e
        diff = (loss(x.double(), w.double() + step) - loss(x.double(), w.double() - step)) / (2 * e)
        assert abs(diff - float(dw[c])) < 1e-4


def test_no_rows():
    dw = torch.full((64,), 3.0, device="cuda")
    C.ec2moe_rmsnorm_backward(C.BF16, C.BF16, 0, 64, 64, 0, 0, 0, 0, 0, 0, dw)
    assert bool((dw == 0).all())
    dw.fill_(3.0)
    C.ec2moe_rmsnorm_backward(C.BF16, C.BF16, 0, 64, 64, 0, 0, 0, 0, 0, 0, dw, accumulate=1)
    assert bool((dw == 3).all())
    C.ec2moe_rmsnorm(C.BF16, C.BF16, 0, 64, 64, 0, 0, 0, 1e-5, 0, 0, 16)


@pytest.mark.parametrize("rows,cols", [(64, 4096), (3000, 2048), (700, 1040)])
def test_8_bit_rows_are_the_definitions(rows, cols):
    """Of the fp32 sum of a row and its residual every e4m3 value is the definition's in 64 bits (the 64-bit quotients
    themselves are 1e-15 off, and none lies that near to a tie here)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, cols, generator=g, device="cuda")).to(BF)
    r = (torch.randint(-64, 65, (rows, cols), generator=g, device="cuda") / 32).to(BF)
    h = (x.float() + r.float()).double()
    w = 1 + 0.3 * rand(cols, seed=2)
    Q, S = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, -(-cols // 128), device="cuda")
    C.ec2moe_rmsnorm(C.BF16, C.BF16, rows, cols, cols, x, r, w, 1e-5, None, None, None, Q, S)
    hw = torch.nn.functional.pad(h * w.double(), (0, -cols % 128)).view(rows, -1, 128)
    want = ref.to_e4m3(hw / (hw.abs().amax(2, keepdim=True) / 448)).view(rows, -1)[:, :cols]
    assert torch.equal(Q.to(F32).double(), want)
