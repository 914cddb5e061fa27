"""What an optimiser updates: the training block's parameters are the tensors that its calls read."""
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


@pytest.mark.parametrize("cfg", [S.preset("finegrained_bf16", T=100, d=256, d_ff=96, r=0, n_shared=2, d_ff_shared=160, seed=1),
                                 S.preset("mixtral_bf16", T=77, d=512, d_ff=448, r=128, seed=2),
                                 S.preset("switch_bf16", T=130, d=768, d_ff=512, seed=3)], ids=lambda c: c.name)
def test_a_step_of_the_parameters_is_a_step_of_the_block(cfg):
    """After an update in place the block is bit for bit the one that is made of the updated weights."""
    inp = S.make_inputs(cfg, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    norm = 1 + 0.3 * torch.randn(cfg.d, generator=g, device="cuda")
    dY = torch.randn(cfg.T, cfg.d, generator=g, device="cuda").to(torch.bfloat16)
    run = runner.TrainBlockRun(cfg, inp, norm)
    before = run.forward()[1].clone()
    run.backward(dY)
    assert set(run.params) == set(run.grads)
    for n, p in run.params.items():
        assert p.shape == run.grads[n].shape, n
        p.sub_((run.grads[n] * (0.3 * p.float().norm() / run.grads[n].norm())).to(p.dtype))
    p = run.params
    new = dict(inp, W2=p["W2"].clone())
    names = [("up", "1", "3", cfg.d_ff, "")]
    if cfg.n_shared:
        names.append(("ups", "1", "3", cfg.d_ff_shared, "s"))
        new["W2s"] = p["W2s"].clone()
    for name, a, b, f, tail in names:
        new["W" + a + tail] = p[name][:, :f].contiguous()
        if cfg.act == C.SWIGLU:
            new["W" + b + tail] = p[name][:, f:].contiguous()
    if cfg.r:
        new["V_enc"], new["V_dec"] = p["V_enc"].clone(), p["V_dec"].clone()
    other = runner.TrainBlockRun(cfg, new, p["norm"].clone())
    Y = run.forward()[1]
    assert torch.equal(other.forward()[1], Y) and not torch.equal(Y, before)
    assert torch.equal(other.backward(dY), run.backward(dY))
    for n in run.grads:
        assert torch.equal(other.grads[n], run.grads[n]), n
    assert C.ec2moe_last_device_error() == C.OK
