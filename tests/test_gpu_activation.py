"""The experts' activation with the gate weight, and its gradient, against 64 bits.

Errors: SiLU and its derivative through fast exponentials, 2e-6 of themselves for the
arguments here (|u| <= 12: e^|u| within |u| 2^-23 and 2 units of 2^-23, the quotient 2 units); the normal
distribution is within 3e-7; a handful of roundings of 2^-24.  2e-6 of each term's magnitude covers them.
bf16 results are rounded by 2^-8.
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


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def make(rows, cols, dtype, glu, seed=0, pad=8):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return (2 * torch.randn(*shape, generator=g, device="cuda")).clamp(-12, 12).to(dtype)

    uv = rand(rows, (2 if glu else 1) * cols + pad)
    perm = torch.randperm(rows, generator=g, device="cuda").int()
    scale = torch.rand(rows, generator=g, device="cuda")
    return uv, perm, scale, rand(rows, cols)


def near(got, want, dtype, scale):
    err = (got.double() - want).abs()
    bound = HALF[dtype] * want.abs() + 2e-6 * scale + 1e-37
    assert bool((err <= bound).all()), float((err / bound).max())


SHAPES = [(1, 8), (3, 24), (257, 1408), (40, 14336), (1000, 1024), (7, 1000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("glu", [True, False])
@pytest.mark.parametrize("routed", [True, False])
def test_both_directions(rows, cols, dtype, glu, routed):
    uv, perm, scale, dh = make(rows, cols, dtype, glu)
    act, ld = C.SWIGLU if glu else C.GELU, uv.shape[1]
    if not routed:
        perm = scale = None
    u, v = uv[:, :cols], uv[:, cols:2 * cols] if glu else None
    H = torch.empty(rows, cols, dtype=dtype, device="cuda")
    C.ec2moe_activation(CODE[dtype], act, rows, cols, ld, u, v, perm, scale, H)
    a, da_u, da_v = ref.activation(u, v, None)
    s = scale.double()[perm.long()][:, None] if routed else torch.ones(rows, 1, dtype=torch.float64, device="cuda")
    size = (u.double().abs() * (v.double().abs() if glu else 1))  # of what cancels in 1 + erf, 1 - p
    near(H, a * s, dtype, size * s)
    duv = torch.full_like(uv, 5.0)
    H2, d_scale = torch.empty_like(H), torch.full((rows,), 5.0, device="cuda")
    C.ec2moe_activation_backward(CODE[dtype], act, rows, cols, ld, u, v, perm, scale, dh, duv,
                                 duv[:, cols:] if glu else None, H2, d_scale)
    assert C.ec2moe_last_device_error() == C.OK
    near(H2, a * s, dtype, size * s)
    g = dh.double() * s
    near(duv[:, :cols], g * da_u, dtype, g.abs() * (1 + u.double().abs()) * (v.double().abs() if glu else 1))
    if glu:
        near(duv[:, cols:2 * cols], g * da_v, dtype, g.abs() * u.double().abs())
    assert bool((duv[:, (2 if glu else 1) * cols:] == 5).all())
    want = torch.empty(rows, dtype=torch.float64, device="cuda")
    terms = torch.empty_like(want)
    at = perm.long() if routed else torch.arange(rows, device="cuda")
    want[at], terms[at] = (dh.double() * a).sum(1), (dh.double().abs() * size).sum(1)
    # a thread adds cols / 32 terms in order at most
    assert bool(((d_scale.double() - want).abs() <= (2e-6 + (cols / 32 + 16) * 2.0 ** -24) * terms).all())
    # in place, and without what is optional
    again, dh2 = uv.clone(), dh.clone()
    C.ec2moe_activation_backward(CODE[dtype], act, rows, cols, ld, again, again[:, cols:] if glu else None, perm, scale, dh2,
                                 again, again[:, cols:] if glu else None, dh2, None)
    n = (2 if glu else 1) * cols
    assert torch.equal(again[:, :n], duv[:, :n]) and torch.equal(dh2, H2) and torch.equal(again[:, n:], uv[:, n:])


@pytest.mark.parametrize("glu", [True, False])
def test_gradient_by_differences(glu):
    """Central differences of the 64-bit forward, step 1e-4: e^2 / 6 times third derivatives below 4 |v| |dh|, and fp32."""
    rows, cols, e = 3, 40, 1e-4
    uv, perm, scale, dh = make(rows, cols, F32, glu, seed=3, pad=0)
    duv, d_scale = torch.empty_like(uv), torch.empty(rows, device="cuda")
    act = C.SWIGLU if glu else C.GELU
    C.ec2moe_activation_backward(C.F32, act, rows, cols, uv.shape[1], uv, uv[:, cols:] if glu else None, perm, scale, dh,
                                 duv, duv[:, cols:] if glu else None, None, d_scale)

    def terms(x, sc):
        a = ref.activation(x[:, :cols], x[:, cols:] if glu else None, None)[0]
        return a * sc[perm.long()][:, None] * dh.double()

    base = uv.double()
    for half in range(2 if glu else 1):
        step = torch.zeros_like(base)
        step[:, half * cols:(half + 1) * cols] = e
        diff = (terms(base + step, scale.double()) - terms(base - step, scale.double())) / (2 * e)
        assert float((diff - duv[:, half * cols:(half + 1) * cols].double()).abs().max()) < 2e-4
    for r in range(rows):
        step = torch.zeros(rows, dtype=torch.float64, device="cuda")
        step[r] = e
        diff = (terms(base, scale.double() + step).sum() - terms(base, scale.double() - step).sum()) / (2 * e)
        assert abs(float(diff) - float(d_scale[r])) < 2e-4 * (1 + abs(float(diff)))


def test_large_arguments():
    u = torch.tensor([[-200.0, -89.0, -30.0, 0.0, 30.0, 200.0, 3e38, -3e38]], device="cuda")
    v = torch.ones_like(u)
    H, du, dv = (torch.empty_like(u) for _ in range(3))
    for act in (C.SWIGLU, C.GELU):
        C.ec2moe_activation(C.F32, act, 1, 8, 8, u, v, None, None, H)
        C.ec2moe_activation_backward(C.F32, act, 1, 8, 8, u, v, None, None, v, du, dv, None, None)
        assert torch.equal(H[0, 3:7], u[0, 3:7]) and torch.equal(du[0, 4:7], torch.ones(3, device="cuda"))
        assert float(H[0, :3].abs().max()) < 1e-11 and float(du[0, :3].abs().max()) < 1e-11 and float(du[0, 3]) == 0.5
        assert float(H[0, 7]) == 0 and float(du[0, 7]) == 0


@pytest.mark.parametrize("glu", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_gradients_rows_are_the_forwards(glu, dtype):
    """Bit for bit, infinities and NaN too: u P(u) and u p are inf at inf and NaN (inf times 0) at -inf, in their place only."""
    rows, cols = 5, 200
    uv, perm, scale, dh = make(rows, cols, dtype, glu, seed=9)
    at = {7: float("inf"), 80: float("-inf"), 199: float("nan")}
    for c, x in at.items():
        uv[2, c] = x
    act, ld = C.SWIGLU if glu else C.GELU, uv.shape[1]
    v = uv[:, cols:] if glu else None
    if glu:
        uv[2, cols:2 * cols] = 1.0
    H, H2, duv = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty_like(dh), torch.zeros_like(uv)
    C.ec2moe_activation(CODE[dtype], act, rows, cols, ld, uv, v, perm, scale, H)
    C.ec2moe_activation_backward(CODE[dtype], act, rows, cols, ld, uv, v, perm, scale, dh, duv,
                                 duv[:, cols:] if glu else None, H2, None)
    bits = torch.int16 if dtype == BF else torch.int32
    assert torch.equal(H.nan_to_num(3.0).view(bits), H2.nan_to_num(3.0).view(bits))
    assert float(H[2, 7]) == float("inf") and bool(H[2, [80, 199]].isnan().all())
    for x in (H, duv):
        bad = (~x.isfinite()).nonzero().tolist()
        assert {r for r, _ in bad} == {2} and {c % cols for _, c in bad} <= set(at)


def test_bad_slots_are_skipped_and_reported():
    uv, perm, scale, dh = make(6, 64, BF, True)
    perm = torch.tensor([0, 5, -1, 2, 6, 1], dtype=torch.int32, device="cuda")
    H, duv = torch.full((6, 64), 5.0, dtype=BF, device="cuda"), torch.full_like(uv, 5.0)
    d_scale = torch.full((6,), 5.0, device="cuda")
    ld = uv.shape[1]
    C.ec2moe_activation(C.BF16, C.SWIGLU, 6, 64, ld, uv, uv[:, 64:], perm, scale, H)
    assert C.ec2moe_last_device_error() == C.ERR_INVALID_ARG
    C.ec2moe_activation_backward(C.BF16, C.SWIGLU, 6, 64, ld, uv, uv[:, 64:], perm, scale, dh, duv, duv[:, 64:], None, d_scale)
    assert C.ec2moe_last_device_error() == C.ERR_INVALID_ARG and C.ec2moe_last_device_error() == C.OK
    a = ref.activation(uv[:, :64], uv[:, 64:128], None)[0]
    for r, slot in enumerate(perm.tolist()):
        if 0 <= slot < 6:
            near(H[r], a[r] * float(scale[slot]), BF, (uv[r, :64].double() * uv[r, 64:128].double()).abs())
        else:
            assert bool((H[r] == 5).all()) and bool((duv[r] == 5).all())
    assert bool((d_scale[[3, 4]] == 5).all())
