"""The training block made on one stream and run on another."""
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


def test_joined_weights_are_there_before_another_stream_reads_them():
    cfg = S.preset("finegrained_bf16", T=64, d=256, d_ff=512, r=0, n_shared=1, d_ff_shared=256, seed=3)
    inp = S.make_inputs(cfg, device="cuda")
    inp["mask"] = inp["mask"].cpu()
    norm = torch.ones(cfg.d, device="cuda")
    dY = torch.randn(cfg.T, cfg.d, device="cuda").to(torch.bfloat16)

    def step(run, stream=None):
        run.forward(stream=stream)
        run.backward(dY, stream=stream)
        torch.cuda.synchronize()
        return {"Y": run.Y, "dX": run.dX, **run.grads}

    ref = {n: v.clone() for n, v in step(runner.TrainBlockRun(cfg, inp, norm)).items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # memory that the weights will be joined in: NaN until they are
    spoilt = [torch.full((n,), 0x7FC0, dtype=torch.int16, device="cuda") for n in [128 << 20] + [1 << 19] * 64]
    torch.cuda.synchronize()
    del spoilt
    torch.cuda._sleep(400_000_000)  # the constructor's stream is busy for some tenths of a second
    got = step(runner.TrainBlockRun(cfg, inp, norm), side)
    assert C.ec2moe_last_device_error() == C.OK
    for n, v in ref.items():
        assert torch.equal(got[n], v), n
