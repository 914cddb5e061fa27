"""The normed layer's gate balanced on a batch with a residual."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from paper_2508_06024_gb300 import runner
from paper_2508_06024_gb300 import synth as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def test_rebalance_takes_the_batch_and_its_residual():
    cfg = S.preset("finegrained_bf16", T=300, d=256, d_ff=96, r=0, n_shared=0, seed=5)
    inp = S.make_inputs(cfg, device="cuda")
    norm = torch.ones(cfg.d, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    X, residual = (torch.randn(cfg.T, cfg.d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    run = runner.Fp8LayerRun(cfg, inp, norm_weight=norm)
    run.forward(X, residual=residual)
    first, logits = float(run.balance()), run.logits.clone()
    assert run.rebalance(1, 0.0, X, residual) == [first]
    assert torch.equal(run.logits, logits)
    # without a norm the gate reads X itself
    plain = runner.Fp8LayerRun(cfg, inp)
    plain.forward(X)
    first = float(plain.balance(X))
    assert plain.rebalance(1, 0.0, X) == [first]
    with pytest.raises(ValueError):
        plain.forward(X, residual=residual)
    with pytest.raises(ValueError):
        run.balance(X)
