"""Sizes at the edge of what the norm, the activation and the grouped products take: host code only."""
import pytest

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


@pytest.mark.parametrize("G", [2, 8, 64, 128])
@pytest.mark.parametrize("N,K", [(8, 8), (4096, 4096), (512, 14336)])
def test_products_of_fewer_rows_than_groups_are_planned(G, N, K):
    """The plan goes by the mean length of a group: less than one row here, which is not a sum of no blocks (a
    division by zero, which ends the process on x86)."""
    for rows in {1, G // 2, G - 1, G}:
        assert C.ec2moe_grouped_gemm_workspace_size(G, rows, N, K) >= 0


@pytest.mark.parametrize("back", [False, True])
def test_activation_of_columns_beyond_32_bit_indexes(back):
    """A row's columns are walked in steps of 2048 at most: the step behind the last one stays below 2^31."""
    A = 0x100000  # an aligned address that is never reached

    def status(cols, rows=0):
        more = dict(dH=A, dU=A, dV=A) if back else {}
        fn = C.ec2moe_activation_backward if back else C.ec2moe_activation
        try:
            fn(C.BF16, C.SWIGLU, rows, cols, cols, A, A, None, None, H=A, stream=0, **more)
        except C.Ec2moeError as e:
            return e.status
        return C.OK

    most = 2 ** 31 - 2048 - 8
    assert status(most) == C.OK
    for cols in (most + 8, 2 ** 31 - 8):
        assert status(cols) == C.ERR_UNSUPPORTED
    assert status(2 ** 31 - 8, rows=1) == C.ERR_UNSUPPORTED
