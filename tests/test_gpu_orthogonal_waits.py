"""Orthogonal factors whose copies or products do not come: the bounded waits run
out, and the call ends with the device usable.  The stall is requested through
aloco_test_stall_tile: the first block leaves out the copies of one slot (of a
small matrix: its first products)."""
import time

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


@pytest.mark.parametrize("shape,slot,lost", [((3, 140, 500), 1, 3), ((20, 200, 300), 0, 8),
                                             ((40, 400, 520), 2, 8), ((1, 300, 6000), 2, 1),
                                             ((3, 40, 200), 0, 1), ((3, 40, 900), 0, 1)],
                         ids=["few", "single", "pairs", "parts", "small", "small_cluster"])
def test_what_is_not_nan_is_right(shape, slot, lost):
    """The matrices of the tiles that the block knew of are lost, in part or as a whole;
    no other is, and no element is a number that comes of operands that were not there.
    (A block knows of at most eight tiles: four in its ring, two whose products are not
    done, and two that its threads have in hand.)"""
    x = _batch(shape)
    want = A.orthogonalize(x)
    A.test_stall_tile(slot)
    out = A.orthogonalize(x)
    torch.cuda.synchronize()
    nan = out.isnan()
    assert torch.equal(torch.where(nan, 0, out), torch.where(nan, 0, want))
    assert 1 <= int(nan.flatten(1).any(1).sum()) <= lost


def test_a_late_copy_stays_for_the_call_that_heeds_it():
    """2e8 cycles, 0.1 s at the highest clock."""
    x = _batch((3, 40, 200))
    logits = torch.randn(4, 900, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    t = torch.arange(4, device="cuda")
    want = A.orthogonalize(x), A.token_logprobs(logits, t)
    A.test_stall_tile(-200_000_000)
    first = A.orthogonalize(x)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    logp = A.token_logprobs(logits, t)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 > 0.09
    assert torch.equal(first, want[0]) and torch.equal(logp, want[1])
