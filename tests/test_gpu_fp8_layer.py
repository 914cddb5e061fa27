"""The layer with 8-bit experts and the balance of its gate, composed from the entry
points as a program composes them (runner.Fp8LayerRun), against the 64-bit oracles.

The oracle starts from the decoded rows that the library's own codec gave (the codec
has tests of its own; a rounding of it more or less moves an 8-bit activation by a whole
step), and the quantised activations have to be its bits.  Tolerance behind them: the
layer's bf16 roundings (slot rows, Y) are within the 1e-2 that every bf16 layer is held
to; hidden values that lie near a rounding boundary of e4m3 move by one step, at most
3.6e-3 of the result's norm (see the product's tests)."""
import numpy as np
import pytest
import torch

from oracle import ec2moe_oracle as layer_orc
from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from paper_2508_06024_gb300 import runner
from paper_2508_06024_gb300 import synth as S
from tests.parity import oracle_inputs, rel_fro, routing_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


CONFIGS = [S.preset("switch_bf16", T=300, d_ff=256, k=2, n_groups=4, seed=3),
           S.preset("finegrained_bf16", T=77, d=256, d_ff=272, seed=4, n_shared=1, d_ff_shared=96),
           S.preset("decode_bf16", T=5, d=512, d_ff=640, r=0, seed=5),
           S.preset("tiny_fp32", T=100, seed=6)]


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
def test_layer_with_8_bit_experts(cfg):
    inp = S.make_inputs(cfg, device="cuda")
    run = runner.Fp8LayerRun(cfg, inp)
    y = run.forward().double().cpu().numpy()
    assert C.ec2moe_last_device_error() == C.OK
    ref = layer_orc.layer_forward(oracle_inputs(inp), cfg.n_groups, cfg.k, cfg.act, top_groups=cfg.top_groups)
    routing_check(run.topk_idx.cpu().numpy(), ref)
    # the same layer with quantised activations, weights and hidden rows
    idx = run.topk_idx.cpu().numpy()
    f64 = {n: S.to_f64(v) for n, v in inp.items() if v is not None and n != "mask"}
    x = f64["X"] if not cfg.r else S.to_f64(run.X_hat)
    wide = {n: np.stack([orc.widen(*orc.quantize(w, 128), 128) for w in f64[n].astype(np.float32)])
            for n in ("W1", "W3", "W2") if n in f64}
    perm = np.argsort(idx.reshape(-1), kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(idx.reshape(-1), minlength=cfg.E))])
    q, s = orc.quantize(x.astype(np.float32))
    assert np.array_equal(orc.e4m3_decode(run.Xq.view(torch.uint8).cpu().numpy()), q[perm // cfg.k])
    assert np.array_equal(run.Xs.cpu().numpy(), s[perm // cfg.k])
    rows = orc.widen(q, s)[perm // cfg.k]
    slot = orc.experts(rows, offsets, wide["W1"], wide.get("W3"), wide["W2"], run.topk_w.cpu().numpy(), perm)
    want = slot.reshape(cfg.T, cfg.k, cfg.d).sum(1)
    for j in range(cfg.n_shared):
        u = x @ f64["W1s"][j].T
        want += (orc.silu(u) * (x @ f64["W3s"][j].T) if cfg.act == S.SWIGLU else orc.gelu(u)) @ f64["W2s"][j].T
    err = rel_fro(y, want)
    assert err <= 3.6e-3 + (1e-2 if cfg.dtype == S.BF16 else 0.0), err


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
def test_balance_of_the_layer(cfg):
    """Loss and bias gradients from X: logits within 2^-17 of a row's size move the probabilities by as much."""
    inp = S.make_inputs(cfg, device="cuda")
    run = runner.Fp8LayerRun(cfg, inp)
    run.forward()
    counts = run.counts.clone()
    loss = float(run.balance(coef=0.5))
    assert C.ec2moe_last_device_error() == C.OK
    f64 = {n: S.to_f64(inp[n]) for n in ("X", "W_local", "b_local", "W_global", "b_global")}
    z = f64["X"] @ f64["W_local"].T + f64["b_local"]
    if cfg.n_groups > 1:
        z = np.concatenate([z, f64["X"] @ f64["W_global"].T + f64["b_global"]], 1)
    mask = inp["mask"].cpu().numpy()
    want = orc.balance(z, mask, run.topk_idx.cpu().numpy(), cfg.n_groups, 0.5, top_groups=cfg.top_groups)
    assert torch.equal(run.counts.reshape(-1), counts)  # as the routing counted
    assert np.array_equal(run.counts.cpu().numpy().reshape(-1), want[1][0])
    assert abs(loss - want[0]) <= 1e-4 * want[0]
    d = run.d_logits.double().cpu().numpy()
    scale = np.abs(want[2]).max()
    assert np.abs(d - want[2]).max() <= 1e-4 * scale
    assert np.abs(run.d_bias.double().cpu().numpy() - want[3]).max() <= 1e-4 * np.abs(want[2]).sum(0).max()


def test_rebalancing_evens_the_loads():
    """Steps along the bias gradients lower the loss of a skewed gate under a mask."""
    cfg = S.preset("finegrained_bf16", T=2000, d=256, d_ff=96, r=0, n_shared=0, seed=7)
    run = runner.Fp8LayerRun(cfg, S.make_inputs(cfg, device="cuda"))
    before = run.inp["b_local"]
    losses = run.rebalance(steps=12, rate=2.0)
    run.forward()
    assert float(run.balance()) < 0.8 * losses[0]
    assert losses[0] > 1.2 and torch.equal(before, S.make_inputs(cfg, device="cuda")["b_local"])
    assert C.ec2moe_last_device_error() == C.OK
