"""A training step of the block around the layer (runner.TrainBlockRun) and the normed 8-bit
layer (runner.Fp8LayerRun with a norm), against 64 bits with the routing that the run took.

Each result is a chain of bf16 roundings of 2^-8 at most, whose relative errors add up at
worst: forward the normed rows, codec's two, up rows, hidden rows, slots, output: 7; backward
the same up to the hidden rows (5), the gradients of hidden rows, up rows, slots, their sum,
codec's two and the last: 12.
"""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from paper_2508_06024_gb300 import runner
from paper_2508_06024_gb300 import synth as S

pytestmark = pytest.mark.gpu
EPS = 1e-5
STEP = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


CONFIGS = [S.preset("finegrained_bf16", T=333, d=256, d_ff=96, r=0, n_shared=2, d_ff_shared=160, seed=1),
           S.preset("mixtral_bf16", T=700, d=512, d_ff=448, r=128, seed=2),
           S.preset("switch_bf16", T=1025, d=768, d_ff=512, seed=3),
           S.preset("decode_bf16", T=1, d=256, d_ff=64, r=0, seed=4)]


def rel(got, want):
    return float((got.double() - want).norm() / want.norm().clamp_min(1e-30))


def hidden(cfg, rows, up):
    u = rows @ up.T
    if cfg.act == S.SWIGLU:
        u, v = u.chunk(2, 1)
        return u * torch.sigmoid(u) * v
    return torch.nn.functional.gelu(u)


def gate_weight_scale(cfg, run, p, dY):
    """|a| |dY W2| of every slot: d_topk_w is the inner product of these two rows, of which the run has roundings; by
    Cauchy's inequality an error of e of either's norm moves the product by at most e |a| |dY W2|, however small it is itself."""
    y = run.x.double()
    scale = torch.zeros(cfg.T, cfg.k, dtype=torch.float64, device="cuda")
    for e in range(cfg.E):
        t, s = (run.topk_idx == e).nonzero(as_tuple=True)
        if t.numel():
            scale[t, s] = hidden(cfg, y[t], p["up"][e]).norm(dim=1) * (dY.double()[t] @ p["W2"][e]).norm(dim=1)
    return scale


def block64(cfg, p, x, residual, idx, w):
    """(H, Y) of the block in 64 bits: experts idx [T, k] with weights w; p: the parameters."""
    h = x if residual is None else x + residual
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * p["norm"]
    if cfg.r:
        y = (y @ p["V_enc"].T) @ p["V_dec"].T

    def expert(rows, up, down):
        return hidden(cfg, rows, up) @ down.T

    out = torch.zeros_like(y)
    for e in range(cfg.E):
        t, s = (idx == e).nonzero(as_tuple=True)
        if t.numel():
            out = out.index_add(0, t, w[t, s][:, None] * expert(y[t], p["up"][e], p["W2"][e]))
    for j in range(cfg.n_shared):
        out = out + expert(y, p["ups"][j], p["W2s"][j])
    return h, out


def setup(cfg, with_residual):
    inp = S.make_inputs(cfg, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(cfg.seed + 100)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)

    norm = 1 + 0.3 * torch.randn(cfg.d, generator=g, device="cuda")
    residual = rand(cfg.T, cfg.d) if with_residual else None
    return inp, norm, residual, rand(cfg.T, cfg.d), rand(cfg.T, cfg.d)


def parameters(run):
    p = {"norm": run.norm_weight, "up": run.up, "W2": run.inp["W2"]}
    if run.cfg.n_shared:
        p["ups"], p["W2s"] = run.ups, run.inp["W2s"]
    if run.cfg.r:
        p["V_enc"], p["V_dec"] = run.inp["V_enc"], run.inp["V_dec"]
    return {n: v.double().requires_grad_() for n, v in p.items()}


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
@pytest.mark.parametrize("with_residual", [True, False])
def test_training_step(cfg, with_residual):
    inp, norm, residual, dY, dH = setup(cfg, with_residual)
    run = runner.TrainBlockRun(cfg, inp, norm, EPS)
    H, Y = run.forward(residual=residual)
    dX = run.backward(dY, dH)
    assert C.ec2moe_last_device_error() == C.OK
    p = parameters(run)
    x = inp["X"].double().requires_grad_()
    w = run.topk_w.double().requires_grad_()
    h, y = block64(cfg, p, x, None if residual is None else residual.double(), run.topk_idx.long(), w)
    assert rel(H, h.detach()) <= STEP and rel(Y, y.detach()) <= 7 * STEP
    grads = torch.autograd.grad((y * dY.double()).sum() + (h * dH.double()).sum(), [x, w, *p.values()])
    assert rel(dX, grads[0]) <= 12 * STEP
    scale = gate_weight_scale(cfg, run, {n: v.detach() for n, v in p.items()}, dY)
    assert bool(((run.d_topk_w.double() - grads[1]).abs() <= 12 * STEP * scale).all())
    for name, want in zip(p, grads[2:]):
        assert rel(run.grads[name], want) <= 12 * STEP, name
    # a second micro-batch, added; the same again bit by bit
    before = {n: v.clone() for n, v in run.grads.items()}
    run.forward(residual=residual)
    assert torch.equal(run.backward(dY, dH, accumulate=1), dX)
    for n, v in run.grads.items():
        assert torch.equal(v, before[n] + before[n]), n


def test_two_blocks_in_a_row():
    """Block 2 takes block 1's output and residual stream; gradients through both."""
    cfg = S.preset("finegrained_bf16", T=200, d=256, d_ff=96, r=0, n_shared=0, seed=5)
    inps = [S.make_inputs(cfg.replace(seed=s), device="cuda") for s in (5, 6)]
    _, norm, _, dY, dH = setup(cfg, False)
    a, b = (runner.TrainBlockRun(cfg, i, norm, EPS) for i in inps)
    H1, Y1 = a.forward()
    H2, Y2 = b.forward(X=Y1, residual=H1)
    d = b.backward(dY, dH)
    dX = a.backward(d, d)  # Y1 and H1 are added in block 2: one gradient for both
    assert C.ec2moe_last_device_error() == C.OK
    pa, pb = parameters(a), parameters(b)
    x = inps[0]["X"].double().requires_grad_()
    h1, y1 = block64(cfg, pa, x, None, a.topk_idx.long(), a.topk_w.double())
    h2, y2 = block64(cfg, pb, y1, h1, b.topk_idx.long(), b.topk_w.double())
    want = torch.autograd.grad((y2 * dY.double()).sum() + (h2 * dH.double()).sum(), [x, pa["up"], pb["up"]])
    assert rel(Y2, y2.detach()) <= 14 * STEP
    for got, ref in ((dX, want[0]), (a.grads["up"], want[1]), (b.grads["up"], want[2])):
        assert rel(got, ref) <= 24 * STEP


def test_captured_step_and_eager_one():
    """A step captured into a graph and replayed on new inputs, while another object of the same weights runs eagerly."""
    cfg = CONFIGS[0]
    inp, norm, residual, dY, dH = setup(cfg, True)
    eager, run = (runner.TrainBlockRun(cfg, inp, norm, EPS) for _ in range(2))
    run.forward(residual=residual)
    run.backward(dY, dH)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run.forward(residual=residual)
        run.backward(dY, dH)
    for seed in (7, 8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (residual, dY):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        eager.forward(residual=residual)
        want = eager.backward(dY, dH)
        torch.cuda.synchronize()
        assert torch.equal(run.dX, want) and torch.equal(run.Y, eager.Y) and torch.equal(run.d_topk_w, eager.d_topk_w)
        for n in run.grads:
            assert torch.equal(run.grads[n], eager.grads[n]), n


@pytest.mark.parametrize("n_shared,r", [(2, 0), (0, 0), (1, 64)])
def test_normed_8_bit_layer(n_shared, r):
    """Hidden values near an e4m3 tie move by a step: 3.6e-3 of the norm per product chain (as for
    the layer without a norm); two quantisations of 2^-4 at most, 2.6e-2 on average, in rows and hidden rows;
    weights likewise.  Independent errors add in squares: 3 x 2.6e-2."""
    cfg = S.preset("finegrained_bf16", T=150, d=256, d_ff=272, r=r, n_shared=n_shared, d_ff_shared=96, seed=9)
    inp, norm, residual, _, _ = setup(cfg, True)
    run = runner.Fp8LayerRun(cfg, inp, norm_weight=norm, eps=EPS)
    Y = run.forward(residual=residual)
    assert C.ec2moe_last_device_error() == C.OK
    ref = runner.TrainBlockRun(cfg, inp, norm, EPS)
    h, y = block64(cfg, {n: v.detach() for n, v in parameters(ref).items()}, inp["X"].double(), residual.double(),
                   run.topk_idx.long(), run.topk_w.double())
    assert rel(run.H, h) <= STEP
    assert rel(Y, y) <= 3 * 2.6e-2
    # the layer's own rows, normed beforehand, give the same routed part
    plain = runner.Fp8LayerRun(cfg, inp)
    other = plain.forward(run.Xn)
    if not run.shared8:
        assert torch.equal(other, Y)
    assert torch.equal(plain.slot, run.slot)
    assert float(run.balance()) == float(plain.balance(run.Xn))
