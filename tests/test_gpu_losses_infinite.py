"""The post-training losses where a sum, a ratio or a margin is infinite and the
loss is not: products of 0 and infinity have no place in it.

What is expected comes in float64 from the definitions, with -log sigmoid as
log(1 + exp(-z)), whose value at +inf is 0.  Tolerances as tests/_losses.py
derives them, over the rows whose log-probability is finite."""
import math

import numpy as np
import pytest
import torch

import _losses as L
from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

BOTH = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def _inputs(n, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = (torch.randn(n, V, generator=g, device="cuda") * 2).to(dtype)
    return x, torch.randint(0, V, (n,), generator=g, device="cuda")


def _h(t):
    return t.detach().cpu().double().numpy()


def _row_bound(lp, V):
    """Bound of a finite row's log-probability and of its part in a sum."""
    ok = np.isfinite(lp)
    lp = np.where(ok, lp, 0.0)
    return np.where(ok, L.tol_logp(lp, V) + 4 * L.U * np.abs(lp), 0.0)


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,pairs,V", [(12, 3, 40), (12, 3, 9001), (90, 20, 257), (2100, 2, 33)])
@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_a_banned_token_in_an_answer(n, pairs, V, dtype, eps):
    """A token of logit -inf in a rejected answer: the margin is +inf, and with no
    flipped labels that pair's loss is 0.  In small and in large calls."""
    x, t = _inputs(n, V, dtype, V)
    cu = np.linspace(0, n, 2 * pairs + 1).astype(np.int64)
    at = int(cu[1])                      # the first pair's rejected answer
    x[at, t[at]] = -math.inf
    ref = torch.full((n,), -math.log(V) - 2.0, device="cuda")
    beta = 0.3
    got = A.preference_loss(x, t, torch.tensor(cu, device="cuda"), ref, beta=beta,
                            label_smoothing=eps)
    th = _h(t).astype(np.int64)
    lp, p = L.logprobs(_h(x), th, 1.0)
    assert lp[at] == -math.inf and np.isfinite(np.delete(lp, at)).all()
    d = lp - _h(ref)
    R = np.array([d[a:b].sum() for a, b in zip(cu[:-1], cu[1:])])
    z = beta * (R[0::2] - R[1::2])
    assert z[0] == math.inf and np.isfinite(z[1:]).all()
    each = np.logaddexp(0.0, -z) * (1 - eps) + (eps * np.logaddexp(0.0, z) if eps else 0.0)
    bound = _row_bound(lp, V)
    assert float(got.log_ratios[1]) == -math.inf
    if eps:
        assert float(got.loss) == math.inf
    else:
        L.assert_sum(got.loss, each.mean(), beta * bound / pairs)
    # the gradient: sigmoid(+inf) = 1 in the first pair
    sig = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), 1 - 1 / (1 + np.exp(-np.abs(z))))
    k = np.zeros(n)
    off = np.zeros(n)
    for i in range(2 * pairs):
        sign, q, rows = 1 if i % 2 == 0 else -1, i // 2, slice(cu[i], cu[i + 1])
        k[rows] = sign * (sig[q] - 1 + eps) * beta / pairs
        # a pair's margin moves the coefficient by sigma' <= 1/4
        pair = bound[cu[2 * q]:cu[2 * q + 2]].sum()
        off[rows] = beta / pairs * (beta * (0.25 * pair if np.isfinite(z[q]) else 0.0) + 16 * L.U)
    want = -p * k[:, None]
    want[np.arange(n), th] += k
    one = np.zeros_like(p)
    one[np.arange(n), th] = 1.0
    dp = p * (2 * L.tol_logp(np.log(np.maximum(p, 1e-300)), V))
    tol = 2 * (np.abs(k)[:, None] * dp + off[:, None] * np.abs(one - p)) + \
        (2.0 ** -8 if dtype == torch.bfloat16 else 4 * L.U) * np.abs(want) + 1e-38
    err = np.abs(_h(got.grad) - want)
    assert np.all(err <= tol), float(np.nanmax(err / tol))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_margins_of_minus_infinity_and_of_none(dtype):
    """A banned token in a chosen answer costs infinitely much; one in both
    answers of a pair leaves no margin."""
    x, t = _inputs(4, 500, dtype, 3)
    cu = torch.tensor([0, 2, 4], device="cuda")
    x[1, t[1]] = -math.inf
    for eps in (0.0, 0.2):
        got = A.preference_loss(x, t, cu, label_smoothing=eps)
        assert float(got.loss) == math.inf and not bool(torch.isnan(got.grad).any())
    x[3, t[3]] = -math.inf
    assert math.isnan(float(A.preference_loss(x, t, cu).loss))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,V", [(9, 40), (9, 50001), (2700, 16001)])
def test_a_reference_that_is_only_watched(n, V, dtype):
    """kl_coef = 0 with a reference: the KL sum is reported, here without a finite value (the
    reference far above, and a banned token), and the loss is the policy term
    alone.  In small calls and where the sums take a kernel of their own."""
    x, t = _inputs(n, V, dtype, V)
    x[1, t[1]] = -math.inf
    lp = A.token_logprobs(x, t)
    assert float(lp[1]) == -math.inf
    old = torch.where(torch.isfinite(lp), lp + 0.1, -9.0)
    ref = old.clone()
    ref[2] += 200.0
    adv = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, 0.5)
    w = torch.full((n,), 1.0 / n, device="cuda")
    got = A.policy_loss(x, t, adv, old, w, ref_logp=ref, kl_coef=0.0)
    assert not math.isfinite(float(got.terms[2]))
    exact = L.logprobs(_h(x), _h(t).astype(np.int64), 1.0)[0]
    r = np.exp(exact - _h(old))
    want = (_h(w) * -np.minimum(r * _h(adv), np.clip(r, 0.8, 1.2) * _h(adv))).sum()
    bound = _h(w) * np.abs(_h(adv)) * (r * _row_bound(exact, V) + 32 * L.U * (r + 1.2))
    L.assert_sum(got.terms[0], want, bound)
    assert torch.equal(got.terms[0], got.terms[1])
    alone = A.policy_loss(x, t, adv, old, w)
    assert torch.equal(got.grad, alone.grad) and torch.equal(got.terms[0], alone.terms[0])
    # with a coefficient it counts
    again = A.policy_loss(x, t, adv, old, w, ref_logp=ref, kl_coef=0.1)
    assert not math.isfinite(float(again.terms[0]))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_ratios_beyond_fp32_without_an_advantage(dtype):
    """r A is 0 where the advantage is, also where r = exp(logp - old) leaves
    fp32 (an old policy that all but ruled the token out)."""
    V = 700
    x, t = _inputs(6, V, dtype, 4)
    lp = A.token_logprobs(x, t)
    old, adv = lp.clone(), torch.zeros(6, device="cuda")
    old[:3] -= 200.0
    adv[5] = -0.0
    old[5] -= 150.0
    w = torch.full((6,), 1.0 / 6, device="cuda")
    got = A.policy_loss(x, t, adv, old, w)
    assert not bool(got.terms[:3].any()) and not bool(torch.isnan(got.terms).any())
    assert not bool(got.grad.any())
    # a missing value stays one
    lost = old.clone()
    lost[0] = math.nan
    assert math.isnan(float(A.policy_loss(x, t, adv, lost, w).terms[0]))
