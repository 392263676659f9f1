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


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_autograd_sees_that_the_logits_were_overwritten(loss):
    """Where the operation before the logits saved its result, a backward pass
    through it is refused after the gradient went over the logits."""
    h = torch.randn(4, 300, device="cuda", requires_grad=True)
    t = torch.randint(0, 300, (4,), device="cuda")
    f = torch.ones(4, device="cuda")
    cu = torch.tensor([0, 2, 4], device="cuda")

    def step(over):
        capped = torch.tanh(h)
        kw = {"grad": capped} if over else {}
        if loss == "policy":
            r = A.policy_loss(capped, t, f, -5 * f, f / 4, **kw)
        else:
            r = A.preference_loss(capped, t, cu, **kw)
        return capped, r.grad

    capped, g = step(False)
    capped.backward(g)
    assert bool(h.grad.any())
    capped, g = step(True)
    assert g.data_ptr() == capped.data_ptr()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        capped.backward(g.detach().clone())


def test_what_is_written_counts_as_written():
    """Version counters move with every tensor that a call writes into, and with
    no other."""
    x = torch.randn(4, 300, device="cuda")
    t = torch.randint(0, 300, (4,), device="cuda")
    f = torch.ones(4, device="cuda")
    cu = torch.tensor([0, 2, 4], device="cuda")
    into = torch.empty_like(x)
    flat = torch.empty(2400, device="cuda")
    lst = A.GradList([x, into])
    seen = [x, t, f, cu, into, flat]
    for call, written in (
            (lambda: A.token_logprobs(x, t), []),
            (lambda: A.policy_loss(x, t, f, f, f), []),
            (lambda: A.policy_loss(x, t, f, f, f, grad=into), [into]),
            (lambda: A.policy_loss(x, t, f, f, f, grad=x), [x]),
            (lambda: A.preference_loss(x, t, cu, grad=into), [into]),
            (lambda: A.preference_loss(x, t, cu, grad=x), [x]),
            (lambda: A.grad_norm(lst), []),
            (lambda: A.clip_grads(lst, 1.0, out=flat), [flat]),
            (lambda: A.clip_grads(lst, 1.0), [x, into])):
        before = [v._version for v in seen]
        call()
        moved = [v for v, b in zip(seen, before) if v._version > b]
        assert [id(v) for v in moved] == [id(v) for v in written]


def test_inference_tensors():
    """They have no version counter, and are taken as before."""
    with torch.inference_mode():
        x = torch.randn(4, 300, device="cuda")
        t = torch.randint(0, 300, (4,), device="cuda")
        f = torch.ones(4, device="cuda")
        want = A.policy_loss(x, t, f, f, f).grad.clone()
        assert torch.equal(A.policy_loss(x, t, f, f, f, grad=x).grad, want)
        lst = A.GradList([x])
        flat = torch.empty(1200, device="cuda")
        A.clip_grads(lst, 1.0, out=flat)
        A.clip_grads(lst, 1.0)
        assert torch.equal(x.reshape(-1), flat)
