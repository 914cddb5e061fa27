"""Which batches the balance loss does in one launch, and that the forms on both sides of
the limit agree: a batch at the limit against the same one with a token more that does not
count (sums in another order: a few units of fp32's last place of the largest term)."""
import numpy as np
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def call(T, E, K, k, z, idx, valid=None):
    desc = C.make_desc(T=T, d=8, E=E, d_ff=0, k=k, n_groups=K)
    wsb = C.ec2moe_balance_loss_workspace_size(desc, 1)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = [torch.empty(1, device="cuda"), torch.empty(1, E, dtype=torch.int32, device="cuda"), torch.empty_like(z),
           torch.empty(z.shape[1], device="cuda")]
    C.ec2moe_balance_loss(desc, z, z.shape[1], np.ones(E, np.uint8), idx, valid, None, 1, 0.5, None, *out, ws, wsb)
    n = C.ec2moe_last_launch_count()
    assert C.ec2moe_last_device_error() == C.OK
    return n, out


# lanes: 131072 logits; rows in shared memory: 1024 tokens; either: 16384 entries
@pytest.mark.parametrize("T,E,K,k", [(131072 // 144, 128, 16, 1), (131072 // 72, 64, 8, 6), (8192, 16, 1, 1), (1024, 96, 12, 6),
                                     (1024, 10, 5, 2), (2048, 8, 1, 8)])
def test_forms_agree_at_the_limit(T, E, K, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    O = E + (K if K > 1 else 0)
    z = torch.randn(T + 1, O, generator=g, device="cuda")
    idx = torch.rand(T + 1, E, generator=g, device="cuda").topk(k, 1).indices.int().contiguous()
    valid = torch.ones(T + 1, dtype=torch.uint8, device="cuda")
    valid[T] = 0
    n, one = call(T, E, K, k, z[:T].contiguous(), idx[:T].contiguous())
    assert n == 1
    n, many = call(T + 1, E, K, k, z, idx, valid)
    assert n == 4
    assert torch.equal(one[1], many[1])
    assert not many[2][T].any()
    assert torch.allclose(one[0], many[0], rtol=1e-5, atol=0)
    assert (one[2] - many[2][:T]).abs().max() <= 1e-5 * one[2].abs().max()
    assert (one[3] - many[3]).abs().max() <= 1e-5 * one[2].abs().sum(0).max()


@pytest.mark.parametrize("T,E,K", [(16384, 128, 16), (16384, 64, 8), (2048, 96, 12)])
def test_long_batches_of_one_expert_per_token_use_the_whole_gpu(T, E, K):
    z = torch.randn(T, E + K, device="cuda")
    idx = torch.randint(0, E, (T, 1), dtype=torch.int32, device="cuda")
    assert call(T, E, K, 1, z, idx)[0] == 4
