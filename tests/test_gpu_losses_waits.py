"""The post-training losses' row kernels when a copy never comes: every wait is
bounded, so the kernels end, NaN stands where it concerns, and the device stays
usable.  The stall is requested through aloco_test_stall_tile: the producer
leaves out one slot's copy, whose barrier is then never completed."""
import time

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu


def _inputs(n, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(n, V, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    f = lambda s: torch.randn(n, generator=g, device="cuda") * s
    return x, t, f(1.0), f(0.1) - 10.0, torch.full((n,), 1.0 / n, device="cuda")


@pytest.mark.parametrize("V,slot,dtype", [(32000, 2, torch.bfloat16), (128256, 1, torch.bfloat16),
                                          (4000, 1, torch.float32)])
def test_a_copy_that_never_comes(V, slot, dtype):
    """One slot of block 0 is never filled: the waits run out, the loss and the
    rows concerned are NaN, every kernel ends and the next call is right."""
    x, t, adv, old, w = _inputs(700, V, dtype, V)
    call = lambda: A.policy_loss(x, t, adv, old, w, ref_logp=old, kl_coef=0.1)
    want = [v.clone() for v in call()]
    torch.cuda.synchronize()
    A.test_stall_tile(slot)
    t0 = time.time()
    got = call()
    torch.cuda.synchronize()
    assert 1.0 < time.time() - t0 < 40.0
    assert bool(torch.isnan(got.terms[:3]).all())
    bad = torch.isnan(got.logp)
    assert 0 < int(bad.sum()) < 350
    assert torch.equal(got.logp[~bad], want[1][~bad])
    assert torch.equal(got.grad[~bad], want[2][~bad])
    again = call()
    assert all(torch.equal(p, q) for p, q in zip(again, want))


def test_a_copy_that_never_comes_in_the_preference_loss():
    x, t, _, old, _ = _inputs(200, 50257, torch.float32, 5)
    cu = torch.tensor([0, 50, 100, 150, 200], device="cuda")
    want = A.preference_loss(x, t, cu, old)
    torch.cuda.synchronize()
    A.test_stall_tile(0)
    got = A.preference_loss(x, t, cu, old)
    torch.cuda.synchronize()
    assert bool(torch.isnan(got.loss)) and bool(torch.isnan(got.logp[0]))
    assert torch.equal(A.preference_loss(x, t, cu, old).grad, want.grad)
