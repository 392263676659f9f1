"""Orthogonal factors whose copies or products do not come: the bounded waits run
out, and the call ends with the device usable.  The stall is requested through
aloco_test_stall_tile: the first block leaves out the copies of one slot (of a
small matrix: its first products)."""
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from _orthogonal import momentum_like

pytestmark = pytest.mark.gpu


def _batch(shape):
    return torch.stack([momentum_like(*shape[1:], torch.Generator("cuda").manual_seed(i))
                        for i in range(shape[0])])


@pytest.mark.parametrize("shape,slot", [((3, 140, 500), 2), ((40, 400, 520), 0), ((30, 768, 768), 40)],
                         ids=["single", "pairs", "pairs_later"])
def test_copies_in_flight_land_before_their_block_ends(shape, slot):
    """The block that gives up fills a ring that its pair and its own threads had
    filled in part.  What follows at once takes the same shared memory and
    accumulators, in this call and in the next ones.  (Slots that the first block fills
    whichever tiles it gets: a tile has three at least, and 41 tiles of 12 come on a
    pair in the last case.)"""
    x = _batch(shape)
    want = A.orthogonalize(x)
    torch.cuda.synchronize()
    A.test_stall_tile(slot)
    out = A.orthogonalize(x)
    after = [A.orthogonalize(x) for _ in range(3)]
    torch.cuda.synchronize()
    assert out.isnan().any()
    assert all(torch.equal(a, want) for a in after)
