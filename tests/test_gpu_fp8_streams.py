"""The layer with 8-bit experts made on one stream and run on another."""
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


def test_weights_are_there_before_another_stream_reads_them():
    cfg = S.preset("switch_bf16", T=64, d_ff=256, r=0, seed=3)
    inp = S.make_inputs(cfg, device="cuda")
    inp["mask"] = inp["mask"].cpu()
    first = runner.Fp8LayerRun(cfg, inp)  # kept: its memory holds the weights
    ref = first.forward()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # memory that the weights will be quantised into: e4m3 NaN until they are
    spoilt = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for n in [256 << 20] + [1 << 20] * 64]
    torch.cuda.synchronize()
    del spoilt
    torch.cuda._sleep(400_000_000)  # the constructor's stream is busy for some tenths of a second
    run = runner.Fp8LayerRun(cfg, inp)
    y = run.forward(stream=side)
    torch.cuda.synchronize()
    assert C.ec2moe_last_device_error() == C.OK
    assert torch.equal(y, ref)
