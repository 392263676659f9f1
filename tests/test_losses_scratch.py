"""The scratch that a loss asks for is what its kernels index: for every row a
cluster's part (24 bytes), maximum and 1 / sum (8) and coefficient (4), and 16
bytes behind them."""
import pytest

from paper_2609_36662_gb300 import aloco as A
from paper_2609_36662_gb300 import build as B


@pytest.mark.parametrize("rows", [1, 2, 3, 1000, 2 ** 27 - 1])
def test_scratch_of_a_loss(rows):
    B.build()
    assert A.load().aloco_loss_scratch_bytes(rows) == 36 * rows + 16
