"""What the runner's normed layer and training block refuse, before anything reaches a GPU."""
import pytest
import torch

from paper_2508_06024_gb300 import runner
from paper_2508_06024_gb300 import synth as S


def bare(cls, **attributes):
    """An object without its buffers: a refused call gets no further than its arguments."""
    run = object.__new__(cls)
    for n, v in attributes.items():
        setattr(run, n, v)
    return run


def test_a_residual_without_a_norm():
    run = bare(runner.Fp8LayerRun, norm_weight=None)
    with pytest.raises(ValueError, match="residual"):
        run.forward(torch.zeros(4, 8), residual=torch.zeros(4, 8))


def test_balance_of_other_rows_than_the_normed_ones():
    run = bare(runner.Fp8LayerRun, norm_weight=torch.ones(8))
    with pytest.raises(ValueError, match="normed"):
        run.balance(torch.zeros(4, 8))


CFG = S.preset("finegrained_bf16", T=4, d=64, d_ff=32, r=0)


@pytest.mark.parametrize("weight", [torch.ones(64, dtype=torch.bfloat16), torch.ones(1).expand(64), torch.ones(32)])
@pytest.mark.parametrize("cls", [runner.Fp8LayerRun, runner.TrainBlockRun])
def test_norm_weights_that_are_not_dense_fp32(cls, weight):
    with pytest.raises(ValueError, match="norm's weight"):
        cls(CFG, {}, norm_weight=weight)


GOOD = torch.zeros(4, 64, dtype=torch.bfloat16)
BAD_ROWS = {
    "type": torch.zeros(4, 64),
    "fewer": torch.zeros(3, 64, dtype=torch.bfloat16),
    "expanded": torch.zeros(1, dtype=torch.bfloat16).expand(4, 64),
    "transposed": torch.zeros(64, 4, dtype=torch.bfloat16).T,
    "device": torch.zeros(4, 64, dtype=torch.bfloat16, device="meta"),
}


@pytest.mark.parametrize("rows", BAD_ROWS.values(), ids=BAD_ROWS)
def test_rows_that_are_not_dense(rows):
    made = dict(cfg=CFG, inp={"X": GOOD}, desc=None, workspace=GOOD, grads={}, Y=GOOD, norm_weight=torch.ones(64))
    block, layer = bare(runner.TrainBlockRun, **made), bare(runner.Fp8LayerRun, **made)
    for call in (lambda: block.forward(rows), lambda: block.forward(residual=rows), lambda: block.backward(rows),
                 lambda: block.backward(GOOD, rows), lambda: layer.forward(rows), lambda: layer.forward(residual=rows)):
        with pytest.raises(ValueError, match="is dense"):
            call()


@pytest.mark.parametrize("cls", [runner.Fp8LayerRun, runner.TrainBlockRun])
def test_a_norm_weight_in_host_memory(cls):
    with pytest.raises(ValueError, match="on cuda"):
        cls(CFG, {}, norm_weight=torch.ones(64))
