"""Lists of gradients whose owners let go of them (as zero_grad() does unless it
is told to keep them), and what the operators write into tensors that autograd
watches."""
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu


def _model(seed=0):
    torch.manual_seed(seed)
    return torch.nn.Sequential(torch.nn.Linear(40, 30), torch.nn.Linear(30, 7)).cuda()


def _backward(m, scale):
    (m(torch.ones(5, 40, device="cuda")) * scale).sum().backward()


def _grads(m):
    return [p.grad for p in m.parameters()]


def _norm(m):
    return float(torch.cat([g.reshape(-1) for g in _grads(m)]).double().norm())


@pytest.mark.parametrize("kept", [False, True])
def test_gradients_that_were_made_anew_are_not_taken_for_the_old(kept):
    """The usual loop drops the gradients and makes others; a list of the old
    ones (which the caller may still hold too) is refused, not answered."""
    m = _model()
    _backward(m, 1.0)
    hold = _grads(m) if kept else None
    lst = A.GradList(_grads(m))
    flat = torch.empty(lst.numel, device="cuda")
    assert float(A.clip_grads(lst, 1e-3, out=flat)) == pytest.approx(_norm(m), rel=1e-5)
    m.zero_grad()
    _backward(m, 3.0)
    for call in (lambda: A.clip_grads(lst, 1e-3, out=flat), lambda: A.grad_norm(lst),
                 lambda: A.clip_grads(lst, 1e-3)):
        with pytest.raises(ValueError, match="anew"):
            call()
    assert float(A.grad_norm(_grads(m))) == pytest.approx(_norm(m), rel=1e-5)
    again = A.GradList(_grads(m))
    assert float(A.grad_norm(again)) == pytest.approx(_norm(m), rel=1e-5)
    assert hold is None or len(hold) == 4


def test_one_gradient_that_was_made_anew():
    m = _model()
    _backward(m, 1.0)
    lst = A.GradList(_grads(m))
    A.clip_grads(lst, 1e-3)
    list(m.parameters())[2].grad = None
    m.zero_grad(set_to_none=False)
    _backward(m, 2.0)
    with pytest.raises(ValueError, match="anew"):
        A.clip_grads(lst, 1e-3)


def test_a_list_made_ahead_of_the_loop():
    m = _model()
    _backward(m, 1.0)
    lst = A.GradList(_grads(m))
    m.zero_grad()
    _backward(m, 2.0)
    with pytest.raises(ValueError, match="anew"):
        A.clip_grads(lst, 1e-3)


def test_gradients_that_stay_are_followed():
    m = _model()
    _backward(m, 1.0)
    lst = A.GradList(_grads(m))
    for scale in (2.0, 5.0, 0.5):
        m.zero_grad(set_to_none=False)
        _backward(m, scale)
        want = _norm(m)
        assert float(A.grad_norm(lst)) == pytest.approx(want, rel=1e-5)
        assert float(A.clip_grads(lst, 1e-3)) == pytest.approx(want, rel=1e-5)
        assert _norm(m) == pytest.approx(1e-3, rel=1e-4)


def test_tensors_that_the_caller_keeps_and_gradients_taken_over():
    """No refusal where a view of a buffer goes and the buffer is written on, nor
    where the caller has taken the gradients from the parameters."""
    flat = torch.ones(1000, device="cuda")
    view = flat.view(10, 100)
    lst = A.GradList([flat])
    assert float(A.grad_norm(lst)) == pytest.approx(1000 ** 0.5, rel=1e-6)
    del view
    flat.fill_(2.0)
    for _ in range(2):
        assert float(A.grad_norm(lst)) == pytest.approx(2 * 1000 ** 0.5, rel=1e-6)
    m = _model()
    _backward(m, 1.0)
    want = _norm(m)
    taken = _grads(m)
    m.zero_grad()
    lst = A.GradList(taken)
    for _ in range(2):
        assert float(A.grad_norm(lst)) == pytest.approx(want, rel=1e-5)
