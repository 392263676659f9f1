"""The float64 losses that the GPU tests compare with, against differences of
their own values and against torch's autograd (CPU)."""
import numpy as np
import pytest
import torch

import _losses as L


def _rows(n, V, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2, (n, V))
    t = rng.integers(0, V, n)
    t[1] = -1
    return rng, x, t


def _policy_args(rng, x, t, tau):
    lp, _ = L.logprobs(x, np.maximum(t, 0), tau)
    n = len(t)
    w = rng.uniform(0.1, 1, n)
    w[2] = 0.0
    return dict(adv=rng.normal(0, 1, n), old=lp + rng.normal(0, 0.4, n), w=w / w.sum(),
                ref=lp + rng.normal(0, 0.4, n), lo=0.2, hi=0.3, kl=0.1, tau=tau)


@pytest.mark.parametrize("tau", [1.0, 0.6])
@pytest.mark.parametrize("V", [2, 9, 40])
def test_policy_gradient_against_differences_and_autograd(V, tau):
    rng, x, t = _rows(7, V, V)
    a = _policy_args(rng, x, t, tau)
    o = L.policy(x, t, **a)
    D, h = rng.normal(0, 1, x.shape), 1e-5
    up, down = L.policy(x + h * D, t, **a), L.policy(x - h * D, t, **a)
    diff = (up["terms"][0] - down["terms"][0]) / (2 * h)
    assert diff == pytest.approx((o["grad"] * D).sum(), rel=1e-6, abs=1e-9)

    q = {k: torch.tensor(v) for k, v in a.items()}
    xt = torch.tensor(x, requires_grad=True)
    tt = torch.tensor(t).clamp(min=0)
    lp = torch.log_softmax(xt / tau, -1).gather(-1, tt[:, None])[:, 0]
    r = torch.exp(lp - q["old"])
    gain = -torch.minimum(r * q["adv"], r.clamp(0.8, 1.3) * q["adv"])
    d = q["ref"] - lp
    live = torch.tensor(t >= 0)
    loss = (torch.where(live, q["w"], 0.0) * (gain + 0.1 * (torch.exp(d) - d - 1))).sum()
    loss.backward()
    assert float(loss) == pytest.approx(o["terms"][0], rel=1e-12)
    assert np.allclose(xt.grad.numpy(), o["grad"], rtol=1e-10, atol=1e-14)


@pytest.mark.parametrize("eps", [0.0, 0.2])
@pytest.mark.parametrize("V", [2, 31])
def test_preference_gradient_against_differences_and_autograd(V, eps):
    rng, x, t = _rows(12, V, 50 + V)
    ref = rng.normal(-2, 1, 12)
    cu = [0, 3, 3, 7, 11]  # one empty sequence, one row of no sequence
    o = L.preference(x, t, cu, ref, 0.3, eps, 0.8)
    D, h = rng.normal(0, 1, x.shape), 1e-5
    diff = (L.preference(x + h * D, t, cu, ref, 0.3, eps, 0.8)["loss"] -
            L.preference(x - h * D, t, cu, ref, 0.3, eps, 0.8)["loss"]) / (2 * h)
    assert diff == pytest.approx((o["grad"] * D).sum(), rel=1e-6, abs=1e-9)
    assert not o["grad"][11].any() and not o["grad"][1].any()

    xt = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(xt / 0.8, -1).gather(-1, torch.tensor(t).clamp(min=0)[:, None])[:, 0]
    d = torch.where(torch.tensor(t >= 0), lp - torch.tensor(ref), 0.0)
    R = torch.stack([d[a:b].sum() for a, b in zip(cu[:-1], cu[1:])])
    z = 0.3 * (R[0::2] - R[1::2])
    near = torch.nn.functional.logsigmoid
    loss = -((1 - eps) * near(z) + eps * near(-z)).mean()
    loss.backward()
    assert float(loss) == pytest.approx(o["loss"], rel=1e-12)
    assert np.allclose(xt.grad.numpy(), o["grad"], rtol=1e-9, atol=1e-14)


def test_a_planted_error_is_seen():
    """The comparison refuses a gradient whose target entry is left out, one of
    the wrong sign and a logp that is off by 1e-4."""
    rng, x, t = _rows(5, 33, 4)
    o = L.policy(x, t, **_policy_args(rng, x, t, 1.0))
    L.assert_grad(o["grad"].astype(np.float32), o, t, False)
    L.assert_logp(o["logp"].astype(np.float32), o["logp"], 33, o["live"])
    wrong = o["grad"].copy()
    wrong[0, t[0]] = -o["coef"][0] * o["p"][0, t[0]]
    for bad in (wrong, -o["grad"]):
        with pytest.raises(AssertionError):
            L.assert_grad(bad, o, t, True)
    with pytest.raises(AssertionError):
        L.assert_logp(o["logp"] + 1e-4 * o["live"], o["logp"], 33)


def test_the_comparison_takes_special_rows():
    """Rows with infinities and NaN, in rows that take part and in others: the
    float64 result passes against itself, and NaN in the wrong place does not."""
    rng, x, t = _rows(7, 20, 9)
    x[3], x[4, 5], x[5, 6] = -np.inf, np.nan, -np.inf
    x[1], x[2], t[5], t[6] = np.nan, np.nan, 6, 20
    a = _policy_args(rng, np.nan_to_num(x, nan=0.0, neginf=0.0), np.minimum(t, 19), 1.0)
    o = L.policy(x, t, **a)
    assert np.isinf(o["logp"][5]) and np.isnan(o["logp"][[3, 4, 6]]).all()
    L.assert_grad(o["grad"], o, t, False)
    L.assert_logp(o["logp"], o["logp"], 20, o["live"])
    L.assert_terms(o["terms"], o)
    wrong = o["grad"].copy()
    wrong[1, 3] = np.nan
    with pytest.raises(AssertionError):
        L.assert_grad(wrong, o, t, False)
    wrong = o["grad"].copy()
    wrong[4, 3] = 0.0
    with pytest.raises(AssertionError):
        L.assert_grad(wrong, o, t, False)
