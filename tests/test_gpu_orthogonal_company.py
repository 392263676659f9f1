"""Whether a matrix takes two steps at a time, and so its factor's precision, does not
depend on what else a call holds: whatever matrices, replicas or passes are beside it."""
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from _orthogonal import COEFFICIENTS, allowed, momentum_like

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = torch.finfo(BF16).eps / 2


def _gen(seed=0):
    return torch.Generator("cuda").manual_seed(seed)


def _batch(n, r, c):
    return torch.stack([momentum_like(r, c, _gen(i)) for i in range(n)])


@pytest.mark.parametrize("shape", [(512, 2048), (1040, 512), (300, 520)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_and_half_of_them(shape):
    """Enough of them in either call that tiles are shared and laid out alike: the same
    bits."""
    x = _batch(90, *shape)
    all_, some = A.orthogonalize(x), A.orthogonalize(x[:45])
    assert torch.equal(all_[:45], some)


@pytest.mark.parametrize("pdt", [F32, BF16], ids=["f32", "bf16"])
def test_replicas(pdt):
    """One replica's step, alone, with others and with other matrices: each within what
    the form of its shape may be off; and as many replicas again change no bit of a replica."""
    r, c, lr = 512, 2048, 2e-2
    n, parts = 2 * r * c, [(0, r, c), (r * c, r, c)]
    x = [(0.02 * torch.randn(n, generator=_gen(i), device="cuda")).to(pdt) for i in range(60)]
    g = [_batch(2, r, c).reshape(-1).roll(i).to(BF16) for i in range(60)]
    cfg = A.muon_cfg(lr=lr, weight_decay=0.0)

    def step(M, parts):
        xs = [t.clone() for t in x[:M]]
        bs = [torch.zeros(n, device="cuda") for _ in xs]
        A.muon_step(xs, g[:M], bs, parts, cfg)
        return xs

    many = step(15, parts)
    more = step(30, parts)
    assert all(torch.equal(a, b) for a, b in zip(many, more))
    u = (1.95 * g[0].double())[:r * c].view(r, c)
    e, off = allowed(u, two_at_a_time=pdt is BF16)
    want = x[0][:r * c].double() - lr * 0.2 * c**0.5 * e.reshape(-1)
    half = torch.finfo(pdt).eps / 2
    tol = lr * 0.2 * c**0.5 * (off + 3 * 2.0**-24 * 485 * float(e.norm())) + \
        (half + 3 * 2.0**-24) * float(want.norm())
    for got in (many[0], step(1, parts)[0], step(1, parts[:1])[0], step(7, parts[:1])[0]):
        assert float((got[:r * c].double() - want).norm()) <= tol


@pytest.mark.parametrize("steps", [1, 2, 3, 5])
@pytest.mark.parametrize("shape", [(3, 512, 1600), (2, 700, 1300), (1, 2200, 520), (12, 800, 1300),
                                   (1, 1030, 1560)], ids=lambda s: "x".join(map(str, s)))
def test_two_steps_at_a_time(shape, steps):
    x = _batch(*shape)
    if shape[0] > 2:
        x[0] = torch.randn(shape[1:], generator=_gen(50), device="cuda")
        x[1] = 0
        x[2, 5, 5] = float("nan")
    for coefficients in ([COEFFICIENTS] * steps,
                         [(3.9, -6.2, 2.6), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0),
                          (1.2, -0.2, 0.0)][:steps]):
        out = A.orthogonalize(x, coefficients=coefficients)
        if shape[0] > 2:
            assert (out[1] == 0).all() and out[2].isnan().all()
        for i in {0, shape[0] - 1} - ({2} if shape[0] > 2 else set()):
            e, tol = allowed(x[i], coefficients=coefficients, two_at_a_time=True)
            assert float((out[i].double() - e).norm()) <= tol + HALF * float(e.norm())
