"""The activation of fp32 rows to fp32's own accuracy, over the arguments at which e^-u is finite.

With e = 2^-24, SwiGLU's errors relative to the result: the exponential 2 units of its last place
(4 e), 1 + e^-u, the quotient, and the three products behind it e each: 9 e.  The derivative is p D, D = 1 +
u (1 - p): p is 6 e off, 1 - p by 6 e p + e (1 - p), D by |u| times that and e |D|, so with |D| <= 1 + |u| and the
three products 17 e p (1 + |u|).  One e more for what is of second order.

GELU is u P(u), P of the fitted complement q = erfc(|u| / sqrt 2) / 2: the fit 1.4e-8, q's own error 16 e
relative for its reciprocal, polynomial and exponential and 1.5 e u^2 for the exponent's rounding.  |u| q <= 0.17 and
|u|^3 q <= 0.23: 2.5e-7 in all, and the result's last roundings, 2 e relative.  The derivative P + u e^(-u^2 / 2) / sqrt(2 pi)
has q <= 0.5 at that error, and the second term's 5 e of 0.25: 7e-7 with its roundings.
"""
import math

import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests import train_reference as ref

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def run(act, u, v, w, dh):
    rows, cols = u.shape
    H, H2, du, dv = (torch.empty_like(u) for _ in range(4))
    C.ec2moe_activation(C.F32, act, rows, cols, cols, u, v, None, w, H)
    C.ec2moe_activation_backward(C.F32, act, rows, cols, cols, u, v, None, w, dh, du, dv, H2, None)
    assert C.ec2moe_last_device_error() == C.OK and torch.equal(H, H2)
    return H.double(), du.double(), dv.double()


def make(most):
    g = torch.Generator(device="cuda").manual_seed(5)
    rows, cols = 64, 2048
    u = (torch.rand(rows, cols, generator=g, device="cuda") * 2 - 1) * most
    u[:32] = 2 * torch.randn(32, cols, generator=g, device="cuda")
    v, dh = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(2))
    return u, v, 0.1 + torch.rand(rows, generator=g, device="cuda"), dh


def test_swiglu():
    u, v, w, dh = make(86.0)
    H, du, dv = run(C.SWIGLU, u, v, w, dh)
    s = w.double()[:, None]
    a, da, db = ref.activation(u, v, None)
    assert bool(((H - a * s).abs() <= 10 * E * (a * s).abs() + 1e-37).all())
    g = dh.double() * s
    assert bool(((dv - g * db).abs() <= 10 * E * (g * db).abs() + 1e-37).all())
    size = torch.sigmoid(u.double()) * (1 + u.double().abs()) * (g * v.double()).abs()
    assert bool(((du - g * da).abs() <= 18 * E * size + 1e-37).all())


def test_gelu():
    u, _, _, _ = make(12.0)
    one = torch.ones(64, device="cuda")
    H, du, _ = run(C.GELU, u, None, one, torch.ones_like(u))
    # the reference's 1 - erf loses nothing in 64 bits; e^(-u^2 / 2) of u to the last bit
    P = 0.5 * torch.special.erfc(-u.double() * math.sqrt(0.5))
    a = u.double() * P
    assert bool(((H - a).abs() <= 2.5e-7 + 2 * E * a.abs()).all())
    da = P + u.double() * torch.exp(-0.5 * u.double() ** 2) / math.sqrt(2 * math.pi)
    assert bool(((du - da).abs() <= 7e-7).all())
