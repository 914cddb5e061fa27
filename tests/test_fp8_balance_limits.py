"""Sizes at the end of the range: what the kernels' 32-bit indexes cannot take is refused
(CPU only; the addresses are never read)."""
import pytest

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

A = 0x100000
LAST = 0x7FFFFFFF


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def status(fn, *args):
    with pytest.raises(C.Ec2moeError) as e:
        fn(*args)
    return e.value.status


@pytest.mark.parametrize("rows", [LAST, LAST - 1, LAST - 254])
def test_product_rows_whose_last_tile_passes_32_bits(rows):
    """A tile of 256 rows begins at most 255 before the end of the rows and ends behind it."""
    assert status(C.ec2moe_fp8_gemm, 1, rows, 16, 16, A, A, None, A, A, C.BF16, A, 16, A, 0, 0) == C.ERR_UNSUPPORTED
    assert C.ec2moe_fp8_gemm_workspace_size(1, rows, 16, 16) == 0


@pytest.mark.parametrize("rows", [LAST, LAST - 1, LAST - 126])
def test_weight_rows_whose_last_block_passes_32_bits(rows):
    """A block of 128 weight rows begins at most 127 before the end of a matrix and ends behind it."""
    assert status(C.ec2moe_fp8_quantize, C.BF16, 1, rows, 16, 16, A, 128, None, 0, A, A, 0) == C.ERR_UNSUPPORTED


@pytest.mark.parametrize("n_seg", [LAST, (1 << 30) + 1])
def test_segments_whose_search_passes_32_bits(n_seg):
    """The search for a token's segment adds two segment numbers."""
    desc = C.make_desc(T=64, d=256, E=1, d_ff=0, k=1, n_groups=1)
    assert status(C.ec2moe_balance_loss, desc, A, 1, bytes([1]), A, None, A, n_seg, 0.01, None, A, A, None, None, A, 1 << 60,
                  0) == C.ERR_UNSUPPORTED
    assert C.ec2moe_balance_loss_workspace_size(desc, n_seg) == 0
