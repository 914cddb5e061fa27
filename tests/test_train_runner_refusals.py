"""What the runner's normed layer and training block refuse, before anything reaches a GPU."""
import pytest
import torch

from paper_2508_06024_gb300 import runner


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
