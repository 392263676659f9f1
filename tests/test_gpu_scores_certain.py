"""Token scores where one token has all the mass or nearly all of it: what is 0 by
definition is 0, nothing has the wrong sign, and small log-probabilities and
entropies keep their digits."""
import math

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF = math.inf

# by warps, by CTAs, by clusters
SIZES = [(40, 1), (300, 700), (2000, 900), (1, 32000), (300, 32000), (1300, 32000), (1300, 20011)]


def _gen(seed=0):
    return torch.Generator("cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,v", SIZES)
def test_one_legal_token(rows, v, dtype):
    x = torch.full((rows, v), -INF, device="cuda")
    t = torch.randint(0, v, (rows,), generator=_gen(rows), device="cuda")
    x.scatter_(1, t[:, None], torch.empty(rows, 1, device="cuda").uniform_(-20, 20, generator=_gen(1)))
    r = A.token_scores(x.to(dtype), t, top=1, temperature=0.7)
    assert (r.logp == 0).all() and (r.entropy == 0).all() and (r.top_logp == 0).all()
    assert (r.stats[:, 1] == 1).all()


def _certain(rows, v, dtype):
    """Rows whose best token is ahead of all others together by up to 60 in logits."""
    x = 2 * torch.randn(rows, v, generator=_gen(rows), device="cuda")
    t = torch.randint(0, v, (rows,), generator=_gen(1), device="cuda")
    x.scatter_(1, t[:, None], -INF)
    by = torch.empty(rows, device="cuda").uniform_(-1, 60, generator=_gen(2))
    return x.scatter(1, t[:, None], (torch.logsumexp(x.double(), 1) + by).float()[:, None]).to(dtype), t


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,v", SIZES[1:])
def test_nothing_has_the_wrong_sign(rows, v, dtype):
    x, t = _certain(rows, v, dtype)
    r = A.token_scores(x, t, top=2)
    assert (r.logp <= 0).all() and (r.entropy >= 0).all() and (r.top_logp <= 0).all()
    y = x.double()
    lp = torch.log_softmax(y, -1)
    # 1e-5 of the sum of the powers of two, and their weights once more (see
    # test_gpu_scores)
    assert ((r.logp - lp.gather(1, t[:, None])[:, 0]).abs() <= 1e-5).all()
    assert ((r.entropy - torch.special.entr(lp.exp()).sum(1)).abs() <= 2e-5 * (1 + r.entropy)).all()


def _small(x, t):
    """(-log p, H) of the best token's rows, from what the others are to it."""
    d = x.double() - x.double().gather(1, t[:, None])
    d.scatter_(1, t[:, None], -INF)
    w = d.exp()
    z = w.sum(1)
    return torch.log1p(z), torch.log1p(z) - torch.where(w > 0, w * d, 0.0).sum(1) / (1 + z)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,v", [(1, 32000), (300, 32000), (300, 128256), (300, 700),
                                    (2000, 900), (1300, 32000), (1300, 20011)])
def test_small_values_keep_their_digits(rows, v, dtype):
    """Where the others are a sixteenth of the sum at most they are summed without the
    largest: 9e-6 of them (see test_gpu_scores), and in the entropy 2^-22 more for the
    rounding of their powers, which lie 2 at least below the largest's."""
    x, t = _certain(rows, v, dtype)
    r = A.token_scores(x, t)
    logp, h = _small(x, t)
    small = (logp < 0.06) & (logp > 1e-30)
    assert ((-r.logp - logp).abs() <= 1e-5 * logp)[small].all()
    assert ((r.entropy - h).abs() <= 1e-5 * h)[small].all()
    # (to the largest logit, which is another where the token is behind it)
    z = (x.double() - x.double().amax(1, keepdim=True)).exp().sum(1)
    assert ((r.stats[:, 1] - z).abs() <= 1e-5 * z).all()


def test_digits_do_not_depend_on_the_rows_beside():
    """A row alone, and among a thousand others: both within 1e-5 of its definition."""
    x, t = _certain(1300, 32000, BF16)
    among = A.token_scores(x, t)
    for i in range(0, 1300, 100):
        one = A.token_scores(x[i:i + 1], t[i:i + 1])
        logp, h = _small(x[i:i + 1], t[i:i + 1])
        if not 1e-30 < float(logp) < 0.06:
            continue
        for r, k in ((one, 0), (among, i)):
            assert abs(float(r.logp[k]) + float(logp)) <= 1e-5 * float(logp)
            assert abs(float(r.entropy[k]) - float(h)) <= 1e-5 * float(h)
