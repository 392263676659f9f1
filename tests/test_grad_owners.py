"""When a kept list of gradients has gone stale: what its owners have let go of
and nothing has written since (CPU tensors; the rule does not touch the device)."""
import torch

from paper_2609_36662_gb300.aloco import _Owned


def _step(p, scale):
    (p * scale).sum().backward()


def test_a_gradient_that_was_dropped_is_stale_and_stays_so():
    p = torch.nn.Parameter(torch.ones(4))
    _step(p, 1.0)
    for hold in ([p.grad], None):
        o = _Owned([p.grad])
        assert len(o.seen) == 1 and not o.stale() and not o.stale()
        p.grad = None
        _step(p, 2.0)
        assert o.stale() and o.stale()
        del hold


def test_a_gradient_that_is_kept_and_added_to():
    p = torch.nn.Parameter(torch.ones(4))
    _step(p, 1.0)
    o = _Owned([p.grad])
    for _ in range(3):
        assert not o.stale()
        p.grad.zero_()
        _step(p, 3.0)


def test_one_of_many():
    ps = [torch.nn.Parameter(torch.ones(4)) for _ in range(5)]
    for p in ps:
        _step(p, 1.0)
    o = _Owned([p.grad for p in ps])
    assert not o.stale()
    ps[3].grad = None
    assert o.stale()


def test_dropped_before_the_first_call():
    """A list made ahead of a loop that begins with zero_grad()."""
    p = torch.nn.Parameter(torch.ones(4))
    _step(p, 1.0)
    o = _Owned([p.grad])
    p.grad = None
    assert o.stale()


def test_gradients_taken_over_from_their_owner():
    p = torch.nn.Parameter(torch.ones(4))
    _step(p, 1.0)
    taken, p.grad = p.grad, None
    o = _Owned([taken])
    assert not o.stale() and not o.stale()


def test_a_buffer_whose_view_goes_and_that_is_written_on():
    flat = torch.ones(100)
    view = flat.view(10, 10)
    o = _Owned([flat])
    assert not o.stale()
    del view
    flat.mul_(2.0)
    assert not o.stale() and not o.stale()


def test_buffers_and_views_of_the_callers_are_not_watched():
    flat = torch.ones(100)
    assert not _Owned([flat]).seen
    with torch.inference_mode():
        x = torch.ones(4)
        y = x[:2]
        assert not _Owned([x, y]).seen
