"""Post-training losses whose blocks come late: the small calls, which finish
within the row kernel, wait for nobody and leave nothing behind for a replay.

A block comes late through aloco_test_stall_tile with a tile below -1: its first
copy is issued so many cycles after its barrier was armed, within the limit of
every wait unless a test says otherwise."""
import time

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

LATE = 600_000_000   # cycles: 0.3 s or more
BOTH = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def _inputs(n, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(n, V, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    f = lambda s: torch.randn(n, generator=g, device="cuda") * s
    return x, t, f(1.0), f(0.1) - 10.0, torch.full((n,), 1.0 / n, device="cuda")


def _calls(n, V, dtype, seed):
    x, t, adv, old, w = _inputs(n, V, dtype, seed)
    cu = torch.tensor([0, n // 4, n // 2, n // 2 + 1, n], device="cuda")
    return x, (lambda: A.policy_loss(x, t, adv, old, w, ref_logp=old, kl_coef=0.1),
               lambda: A.preference_loss(x, t, cu, old))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,V", [(2, 300), (48, 32000), (700, 4000), (1900, 600), (5, 128256)])
def test_a_block_that_comes_last(n, V, dtype):
    """The same results, bit for bit, when block 0 comes long after all others."""
    _, calls = _calls(n, V, dtype, V)
    for call in calls:
        want = [v.clone() for v in call()]
        torch.cuda.synchronize()
        A.test_stall_tile(-LATE)
        t0 = time.time()
        got = call()
        torch.cuda.synchronize()
        assert 0.1 < time.time() - t0 < 2.0
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_a_captured_call_whose_block_comes_late(dtype):
    """Every replay has the same mark and, here, the same late block: none of them
    takes what an earlier one left for its own."""
    x, calls = _calls(40, 5000, dtype, 7)
    for call in calls:
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        A.test_stall_tile(-LATE)
        with torch.cuda.graph(graph):
            got = call()
        for seed in (1, 2, 3):
            x.copy_(_inputs(40, 5000, dtype, seed)[0])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, call()))


def test_small_calls_many_times_over():
    """Whoever comes last adds: the results do not depend on who it is."""
    for n, V in ((3, 257), (64, 1000), (152, 33), (1216, 40), (300, 32000)):
        _, calls = _calls(n, V, torch.bfloat16, n)
        for call in calls:
            want = [v.clone() for v in call()]
            for _ in range(150):
                assert all(torch.equal(p, q) for p, q in zip(call(), want))


TOO_LATE = 6_000_000_000   # cycles: 3 s, where a wait's limit is about 2


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,V", [(2, 300), (20, 4000), (7, 32000), (3, 128256)])
def test_a_copy_that_comes_too_late_lands_before_its_block_ends(n, V, dtype):
    """The consumers have given up when the copy is issued, and the producer has no
    slot to wait for; the block stays until the copy has landed (else the row's
    log-probability would read 0), the row is NaN, and the next call is right."""
    x, calls = _calls(n, V, dtype, V)
    t = torch.randint(0, V, (n,), device="cuda")
    for call, logp in ((calls[0], lambda r: r.logp), (calls[1], lambda r: r.logp),
                       (lambda: A.token_logprobs(x, t), lambda r: r)):
        want = logp(call()).clone()
        torch.cuda.synchronize()
        A.test_stall_tile(-TOO_LATE)
        t0 = time.time()
        got = call()
        torch.cuda.synchronize()
        assert 2.0 < time.time() - t0 < 40.0
        assert bool(torch.isnan(logp(got)[0]))
        if not torch.is_tensor(got):
            assert bool(torch.isnan(got[0].reshape(-1)[0]))  # the loss
        bad = torch.isnan(logp(got))
        assert torch.equal(logp(got)[~bad], want[~bad])
        assert torch.equal(logp(call()), want)
