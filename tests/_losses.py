"""The post-training losses and the clipping in float64, from their formulas,
and how far results in fp32 may lie from them.

Tolerances, from u = 2^-24 (half an fp32 step at 1), before any run:
  logp = (x_a - m) / tau - log z.  The difference, its product with 1 / tau,
      the logarithm and the last difference each round once: at most
      4 u (|logp| + log z + 1), with 0 <= log z <= log V.  An exponential is
      off by its function's error (2 steps), by the rounding of its argument
      (at most 1.5 u times the argument, where it still counts below some 20)
      and the sum by the depth of its tree (under 32 additions, of positive
      terms): below 64 u of z.  TOL_LOGP(row) = 4 u (|logp| + log V + 1) + 64 u.
  p_j: relative TOL_LOGP of the row and 2 u (|log p_j| + 1).
  k = dL/dlogp / tau: its derivative by logp times TOL_LOGP, and 16 u of the
      terms it is formed from.
  gradient: |k| dp + |dk| |[j = a] - p| + the store's rounding (2^-9 of the
      value for bf16, u for fp32).
  sums over rows: the rows' errors added up, and u of the result.
Every bound is then doubled.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def logprobs(x, t, tau):
    """(logp, p) of rows x [n, V] (float64) and tokens t [n]; NaN where a token
    is out of the vocabulary.  Negative tokens: logp 0."""
    n, V = x.shape
    y = x / tau
    with np.errstate(all="ignore"):
        m = y.max(-1, keepdims=True) if V else np.zeros((n, 1))
        e = np.exp(y - m)
        z = e.sum(-1, keepdims=True)
        p = e / z
        at = np.clip(t, 0, V - 1)
        lp = (np.take_along_axis(y, at[:, None], 1) - m - np.log(z))[:, 0]
    lp = np.where(t >= V, np.nan, lp)
    return np.where(t < 0, 0.0, lp), p


def by_logits(p, t, coef, live, tau):
    """coef d logp / d logits, zeros in rows that take no part."""
    with np.errstate(all="ignore"):
        g = -p * (coef / tau)[:, None]
        rows = np.nonzero(live & (t < p.shape[1]))[0]
        g[rows, t[rows]] += coef[rows] / tau
    g[~live] = 0.0
    return g


def policy(x, t, adv, old, w, ref, lo, hi, kl, tau):
    """terms [4], logp, gradient, and dL/dlogp with its derivative's size."""
    live = (t >= 0) & (w != 0)
    lp, p = logprobs(x, t, tau)
    with np.errstate(all="ignore"):
        r = np.exp(lp - old)
        free, bound = r * adv, np.clip(r, 1 - lo, 1 + hi) * adv
        act = free <= bound
        d = (ref - lp) if ref is not None else np.zeros_like(lp)
        back = np.exp(d)
        k3 = back - d - 1
        coef = w * (np.where(act | np.isnan(free), -free, 0.0) + kl * (1 - back))
        slope = np.abs(w) * (np.abs(free) + kl * back)
        # each row's error in the two sums: what logp's does, and rounding
        tl, a = tol_logp(lp, x.shape[1]), np.abs(w)
        off_gain = a * (np.abs(free) * tl + 16 * U * (np.abs(free) + np.abs(bound)))
        off_k3 = a * (np.abs(1 - back) * tl + 4 * U * (back + np.abs(d) + 1))
        per = [-np.minimum(free, bound) + kl * k3, -np.minimum(free, bound), k3,
               np.where(act, 0.0, 1.0)]
        terms = np.array([(w * q)[live].sum() for q in per])
    return dict(terms=terms, logp=np.where(live, lp, 0.0), live=live, p=p, coef=coef,
                slope=slope, off=[(off_gain + kl * off_k3)[live], off_gain[live], off_k3[live],
                                  4 * U * a[live]], grad=by_logits(p, t, coef, live, tau), tau=tau)


def preference(x, t, cu, ref, beta, eps, tau):
    live = t >= 0
    lp, p = logprobs(x, t, tau)
    n = len(t)
    d = np.where(live, lp - (ref if ref is not None else 0.0), 0.0)
    cu = np.clip(np.asarray(cu, np.int64), 0, n)
    R = np.array([d[a:b].sum() for a, b in zip(cu[:-1], cu[1:])])
    pairs = len(R) // 2
    z = beta * (R[0::2] - R[1::2])
    with np.errstate(all="ignore"):
        softplus = np.log1p(np.exp(-np.abs(z)))
        loss = (1 - eps) * (softplus + np.maximum(-z, 0)) + eps * (softplus + np.maximum(z, 0))
        sig = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))),
                       np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
    s = (sig - 1 + eps) * beta / max(pairs, 1)
    coef, slope = np.zeros(n), np.zeros(n)
    for k in range(pairs):
        for i, sign in ((0, 1.0), (1, -1.0)):
            a, b = cu[2 * k + i], cu[2 * k + i + 1]
            coef[a:b] = sign * s[k]
            # d coef / d z, times beta for each token's logp
            slope[a:b] = beta * beta / max(pairs, 1) * sig[k] * (1 - sig[k]) * \
                max(1, cu[2 * k + 2] - cu[2 * k])
    return dict(loss=loss.mean() if pairs else 0.0, ratios=R, logp=np.where(live, lp, 0.0),
                live=live, p=p, coef=np.where(live, coef, 0.0), slope=slope,
                grad=by_logits(p, t, coef, live, tau), tau=tau)


def tol_logp(lp, V):
    return 2 * (4 * U * (np.abs(lp) + np.log(V) + 1) + 64 * U)


def assert_logp(got, lp, V, live=None):
    got = np.asarray(got, np.float64).reshape(-1)
    bad = ~np.isfinite(lp)
    assert np.array_equal(np.isnan(got), np.isnan(lp)), "NaN rows of logp"
    assert np.array_equal(got[bad & ~np.isnan(lp)], lp[bad & ~np.isnan(lp)])
    err = np.abs(got[~bad] - lp[~bad])
    assert np.all(err <= tol_logp(lp, V)[~bad]), float(err.max())
    if live is not None:
        assert not np.any(got[~live])


def assert_grad(got, o, t, bf16):
    """`o`: what policy() or preference() gave."""
    got = np.asarray(got, np.float64).reshape(o["grad"].shape)
    want, p, V = o["grad"], o["p"], o["grad"].shape[1]
    assert not np.any(got[~o["live"]]), "rows that take no part"
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN places of the gradient"
    with np.errstate(all="ignore"):
        tl = tol_logp(o["logp"], V)[:, None]
        k = np.abs(o["coef"] / o["tau"])[:, None]
        dk = (o["slope"] / o["tau"])[:, None] * tl + 16 * U * (k + (o["slope"] / o["tau"])[:, None])
        dp = p * (tl + 2 * U * (np.abs(np.log(np.maximum(p, 1e-300))) + 1))
        onehot = np.zeros_like(p)
        rows = np.nonzero(o["live"] & (t < V))[0]
        onehot[rows, t[rows]] = 1.0
        tol = 2 * (k * dp + dk * np.abs(onehot - p)) + \
            (2.0 ** -8 if bf16 else 2 * U) * np.abs(want) + 1e-38
        ok = np.isnan(want) | (got == want) | (np.abs(got - want) <= tol)
    assert np.all(ok), (int((~ok).sum()), np.argwhere(~ok)[:4].tolist(), got[~ok][:4],
                        want[~ok][:4])


def assert_sum(got, want, parts):
    """A sum over rows: `parts`, the rows' own bounds."""
    got, want = float(got), float(want)
    if np.isnan(want):
        assert np.isnan(got)
        return
    assert abs(got - want) <= 2 * (float(np.sum(parts)) + U * abs(want)) + 1e-38, (got, want)


def assert_terms(got, o):
    """The policy loss's four sums (no ratio at an edge of the clipping)."""
    for g, want, parts in zip(got, o["terms"], o["off"]):
        assert_sum(g, want, parts)


def assert_preference(loss, ratios, o, cu, beta, V):
    n = len(o["logp"])
    cu = np.clip(np.asarray(cu, np.int64), 0, n)
    tl = np.where(o["live"], tol_logp(o["logp"], V) + 2 * U * np.abs(o["logp"]), 0.0)
    offs = np.array([tl[a:b].sum() for a, b in zip(cu[:-1], cu[1:])])
    for g, want, off in zip(np.asarray(ratios, np.float64), o["ratios"], offs):
        assert_sum(g, want, off)
    # |dL/dz| <= 1
    assert_sum(loss, o["loss"], beta * offs / max(1, len(offs) // 2))
