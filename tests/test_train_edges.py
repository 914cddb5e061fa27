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
