"""Grouped products of fewer rows than groups, and a training step with fewer routed rows than experts."""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from paper_2508_06024_gb300 import runner
from paper_2508_06024_gb300 import synth as S
from tests.test_gpu_grouped import FORMS, call, check, operands

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("G,rows,N,K", [(8, 4, 264, 520), (8, 1, 4096, 1024), (64, 63, 136, 264), (128, 127, 72, 64)])
@pytest.mark.parametrize("out_type", [C.BF16, C.F32])
def test_products(form, G, rows, N, K, out_type):
    g = torch.Generator().manual_seed(rows)
    offsets = [0, *sorted(torch.randint(0, rows + 1, (G - 1,), generator=g).tolist()), rows]
    X, W = operands(form, rows, N, K, G, seed=4)
    out = call(form, X, W, offsets, G, rows, N, K, out_type)
    check(form, X, W, offsets, G, rows, N, K, out, out_type)


def test_training_step_of_one_token():
    """2 routed rows, 8 experts: the experts that have none get weight gradients of 0."""
    cfg = S.preset("mixtral_bf16", T=1, d=256, d_ff=96, r=0, seed=6)
    assert cfg.T * cfg.k < cfg.E
    run = runner.TrainBlockRun(cfg, S.make_inputs(cfg, device="cuda"), torch.ones(cfg.d, device="cuda"))
    run.forward()
    run.backward(torch.ones(cfg.T, cfg.d, dtype=torch.bfloat16, device="cuda"))
    assert C.ec2moe_last_device_error() == C.OK
    chosen = run.topk_idx[0].tolist()
    for name in ("up", "W2"):
        for e in range(cfg.E):
            assert bool((run.grads[name][e] == 0).all()) == (e not in chosen), (name, e)
