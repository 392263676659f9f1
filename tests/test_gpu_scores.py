"""Token scores and their gradient against their definitions in 64 bits.

Tolerances, for powers of two 2^t with |t| <= 40 where they matter (what is
smaller adds less than V 2^-40): a term is off by 2 ulp of ex2 and by the
rounding of t, 40 ln 2 2^-24; its sum by at most 32 + 32 + 13 additions; log2(e)
/ tau by its rounding.  Together (4 + 28 + 28 + 77) 2^-24 < 9e-6 of the sum, and
with the logarithm 1e-5 on log-probabilities; twice that on p (and on entropies
relative to 1 + H, whose terms have one more factor)."""
import math

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = math.nan, math.inf


def _gen(seed=0):
    return torch.Generator("cuda").manual_seed(seed)


def _logits(rows, v, dtype, seed=0, std=2.0):
    x = torch.randn(rows, v, generator=_gen(seed), device="cuda") * std
    t = torch.randint(0, v, (rows,), generator=_gen(seed + 1), device="cuda")
    x.scatter_add_(1, t[:, None], torch.full((rows, 1), math.log(v), device="cuda"))
    return x.to(dtype), t


def _want(x, t, k, temp=1.0):
    lp = torch.log_softmax(x.double() / temp, -1)
    ids = torch.sort(x.float(), stable=True, dim=-1, descending=True)[1][..., :k]
    return (lp.gather(-1, t.clamp(0)[..., None])[..., 0], torch.special.entr(lp.exp()).sum(-1),
            ids, lp.gather(-1, ids))


def _check(r, x, t, k, temp=1.0):
    logp, h, ids, best = _want(x, t, k, temp)
    live = t >= 0
    logp, h = torch.where(live, logp, 0.0), torch.where(live, h, 0.0)
    assert ((r.logp - logp).abs() <= 1e-5 + logp.abs() * 2.0 ** -22).all()
    assert ((r.entropy - h).abs() <= 2e-5 * (1 + h)).all()
    if k:
        ids = torch.where(live[..., None], ids, -1)
        best = torch.where(live[..., None], best, 0.0)
        assert torch.equal(r.top_ids.long(), ids)
        both = best == -INF
        assert torch.equal(r.top_logp == -INF, both)
        off = (r.top_logp - best).abs()
        assert (off[~both] <= 1e-5 + best[~both].abs() * 2.0 ** -22).all()
    else:
        assert r.top_ids is None and r.top_logp is None


def _check_grad(x, t, k, temp=1.0, seed=5, parts=("logp", "entropy", "top"), grad=None, over=False):
    rows = t.shape
    r = A.token_scores(x, t, top=k, temperature=temp)
    by = {}
    for i, name in enumerate(parts):
        shape = (*rows, k) if name == "top" else rows
        by["d_" + name] = torch.randn(shape, generator=_gen(seed + i), device="cuda")
    y = x.double()
    lp = torch.log_softmax(y / temp, -1)
    p = lp.exp()
    h = torch.special.entr(p).sum(-1, keepdim=True)
    d = torch.zeros_like(p)
    if "logp" in parts:
        d.scatter_add_(-1, t.clamp(0)[..., None], by["d_logp"].double()[..., None])
    if "top" in parts:
        d.scatter_add_(-1, r.top_ids.long().clamp(0), by["d_top"].double())
    total = d.sum(-1, keepdim=True)
    want = d - p * total
    size = p * total.abs()
    if "entropy" in parts:
        e = by["d_entropy"].double()[..., None]
        plogp = torch.special.entr(p)
        want = want + e * (plogp - p * h)
        # log p is off by 1e-5 and H by 2e-5 (1 + H), also where their sum is near 0
        size = size + e.abs() * (plogp + 2 * p * (1 + h))
    live = (t >= 0)[..., None]
    want = torch.where(live, want / temp, 0.0)
    g = A.token_scores_grad(x, t, r, temperature=temp, grad=x if over else grad, **by)
    half = torch.finfo(x.dtype).eps / 2
    # powers of two below 2^-126 are 0: off by them times what multiplies p (90:
    # -log p there)
    flushed = 2.0 ** -125 * (1 + total.abs() + (by["d_entropy"].abs()[..., None] * (h + 90)
                             if "entropy" in parts else 0)) / temp
    mass = (d.abs().sum(-1, keepdim=True) + (by["d_entropy"].abs().double()[..., None] * h
            if "entropy" in parts else 0)) / temp
    tol = (2e-5 * size + 2.0 ** -22 * d.abs()) / temp + p * mass * 34 * 2.0 ** -24 + \
        half * want.abs() + flushed
    off = (g.double() - want).abs()
    assert torch.where(live, off <= tol, g == 0).all(), float((off / tol).max())
    return g


VOCABS = [1, 2, 7, 8, 9, 31, 32, 33, 255, 256, 257, 1000, 2047, 2048, 4095, 8200, 32000, 50257,
          131072, 262143, 262144]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("v", VOCABS)
def test_vocabularies(v, dtype):
    x, t = _logits(5, v, dtype, seed=v)
    t[3] = -1
    for k in sorted({0, 1, min(5, v), min(32, v)}):
        _check(A.token_scores(x, t, top=k), x, t, k)
    _check_grad(x, t, min(5, v), seed=v + 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,v", [(1, 32000), (3, 9000), (40, 30011), (300, 128256), (2000, 513), (1300, 50257)])
def test_tokens_that_are_nearly_certain(rows, v, dtype):
    """log p = -log(1 + r) of the largest has r's own relative error, that of the other
    terms' sum, and the logarithm's; where rows are many also that of at most 60 additions
    behind the largest term and four roundings more, 2^-25 of it each."""
    x = 2 * torch.randn(rows, v, generator=_gen(rows), device="cuda")
    t = torch.randint(0, v, (rows,), generator=_gen(1), device="cuda")
    x.scatter_(1, t[:, None], -INF)
    by = torch.tensor([0.5, 3.0, 8.0, 14.0], device="cuda")[torch.arange(rows, device="cuda") % 4]
    x = x.scatter(1, t[:, None], (torch.logsumexp(x.double(), 1) + by).float()[:, None]).to(dtype)
    r = A.token_scores(x, t, top=2)
    y = x.double()
    d = y - y.gather(1, t[:, None])
    d.scatter_(1, t[:, None], -INF)
    want = -torch.log1p(d.exp().sum(1))
    more = 64 * 2.0**-25 if rows > 1200 else 0.0
    assert ((r.logp - want).abs() <= 1e-5 * want.abs() + more).all()
    assert torch.equal(r.top_logp[:, 0], r.logp) or (r.top_ids[:, 0] != t).any()
    # stats: the same sum, times the largest's term
    assert ((r.stats[:, 1] - want.neg().exp()).abs() <= 1e-5 * want.neg().exp()).all()


@pytest.mark.parametrize("rows", [1, 2, 37, 300, 1300])
@pytest.mark.parametrize("v,dtype", [(9001, BF16), (20011, F32), (129, BF16)])
def test_row_counts(rows, v, dtype):
    x, t = _logits(rows, v, dtype, seed=rows)
    t[::5] = -7
    _check(A.token_scores(x, t, top=20, temperature=0.7), x, t, 20, 0.7)
    _check_grad(x, t, 8, temp=0.7)


@pytest.mark.parametrize("temp", [0.05, 0.7, 1.0, 3.0])
@pytest.mark.parametrize("parts", [("logp",), ("entropy",), ("top",), ("logp", "entropy"),
                                   ("logp", "entropy", "top")], ids="-".join)
def test_gradients_of_each_part(parts, temp):
    x, t = _logits(4, 3001, F32, seed=9)
    _check_grad(x, t, 6, temp, parts=parts)


def test_gradient_against_differences():
    """The loss itself moves as the gradient says, along random directions."""
    x, t = _logits(3, 400, F32, seed=11)
    k = 4
    r = A.token_scores(x, t, top=k)
    a, b = (torch.randn(3, generator=_gen(i), device="cuda") for i in (1, 2))
    c = torch.randn(3, k, generator=_gen(3), device="cuda")
    g = A.token_scores_grad(x, t, r, d_logp=a, d_entropy=b, d_top=c).double()

    def loss(y):
        s = A.token_scores(y, t, top=k)
        lp = torch.log_softmax(y.double(), -1)     # of the same alternatives
        return float((s.logp.double() * a).sum() + (s.entropy.double() * b).sum() +
                     (lp.gather(-1, r.top_ids.long()) * c).sum())

    for seed in range(3):
        d = torch.randn(x.shape, generator=_gen(20 + seed), device="cuda")
        h = 2e-2
        slope = (loss(x + h * d) - loss(x - h * d)) / (2 * h)
        # central differences: third derivatives times h^2, and 3e-5 / h of the losses' error
        assert abs(slope - float((g * d).sum())) <= 2e-2 * (1 + abs(slope))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_layouts(dtype):
    """Views without the last position, position by position, padded rows and
    starts off any boundary, with gradients that lie otherwise."""
    base = torch.randn(4, 7, 1050, generator=_gen(1), device="cuda").to(dtype)
    t = torch.randint(0, 1003, (4, 6), generator=_gen(2), device="cuda")
    for x in (base[:, :-1, :1003], base[:, 1:, 3:1006], base.transpose(0, 1)[:-1, :, 5:1008]):
        tt = t.reshape(x.shape[:2])
        tt = tt.to(torch.int32)
        _check(A.token_scores(x, tt.contiguous(), top=7), x, tt.long(), 7)
        _check_grad(x, tt.long().contiguous(), 7)
        out = torch.full((*x.shape[:2], 1010), 3.0, dtype=dtype, device="cuda")
        _check_grad(x, tt.long().contiguous(), 7, grad=out[..., 4:1007])
        assert (out[..., :4] == 3).all() and (out[..., 1007:] == 3).all()


def test_gradient_over_the_logits():
    for dtype in (F32, BF16):
        x, t = _logits(40, 5003, dtype, seed=3)
        t[7] = -1
        fresh = _check_grad(x.clone(), t, 9)
        g = _check_grad(x, t, 9, over=True)
        assert g is x and torch.equal(g, fresh)


def test_ties_go_to_the_lowest_index():
    v = 40000
    for dtype in (F32, BF16):
        x = torch.zeros(6, v, dtype=dtype, device="cuda")
        x[1] = torch.arange(v, device="cuda").remainder(3).to(dtype)
        x[2, 17::1000] = 4
        x[3, -40:] = 2
        x[4] = torch.finfo(dtype).min
        x[4, 39990] = 1
        x[5, ::2] = -0.0
        t = torch.randint(0, v, (6,), device="cuda", generator=_gen())
        _check(A.token_scores(x, t, top=32), x, t, 32)


def test_many_large_values_in_few_places():
    """Everything worth having lies in a few threads' elements."""
    v = 60000
    for dtype in (F32, BF16):
        x = torch.randn(3, v, generator=_gen(), device="cuda").to(dtype)
        for u in range(4000 // 8):
            at = u * 8 * 256
            if at + 8 <= v:
                x[0, at:at + 8] += 20
        x[1, 100:2100] += 30
        x[2, :] = torch.arange(v, device="cuda").to(dtype)
        t = torch.randint(0, v, (3,), device="cuda", generator=_gen())
        _check(A.token_scores(x, t, top=32), x, t, 32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 33000])
def test_masked_rows(v, dtype):
    low = torch.finfo(dtype).min
    x, t = _logits(8, v, dtype, seed=4)
    x[0, 5:] = -INF
    x[1, : v - 3] = -INF
    x[2, 9:] = low
    x[3, :] = low
    x[4, ::2] = -INF
    x[5, 1:] = -INF
    x[6, : v // 2] = low
    x[6, v // 2:] = -INF
    t[:] = torch.tensor([3, v - 1, 2, 11, 1, 0, 4, 100], device="cuda")
    _check(A.token_scores(x, t, top=16), x, t, 16)
    _check_grad(x, t, 3)


def test_rows_without_a_value():
    x, t = _logits(6, 700, F32, seed=6)
    x[0, 13] = NAN
    x[1, 500] = INF
    x[2] = -INF
    t[4] = 700
    r = A.token_scores(x, t, top=3)
    for bad in range(3):
        assert r.logp[bad].isnan() and r.entropy[bad].isnan()
        assert (r.top_ids[bad] == -1).all() and r.top_logp[bad].isnan().all()
    assert r.logp[4].isnan() and r.entropy[4].isfinite()
    keep = [3, 5]
    _check(A.TokenScores(*[f[keep] for f in r]), x[keep], t[keep], 3)
    one = torch.ones(6, device="cuda")
    g = A.token_scores_grad(x, t, r, d_logp=one, d_entropy=one)
    assert g[[0, 1, 2, 4]].isnan().all() and g[keep].isfinite().all()


def test_logits_of_any_size():
    for scale in (1e3, 1e6, 1e20, 1e37, 1e-20):
        for dtype in (F32, BF16):
            x = (torch.randn(4, 900, generator=_gen(8), device="cuda") * scale).to(dtype)
            t = x.argmax(-1)
            t[0] = 5
            r = A.token_scores(x, t, top=4)
            logp, h, ids, best = _want(x, t, 4)
            assert torch.equal(r.top_ids.long(), ids)
            # y's rounding, 2^-24 of the logits' spread
            tol = 1e-5 + 2.0 ** -21 * logp.abs()
            ok = logp.abs() < 3e38
            assert ((r.logp - logp).abs() <= tol)[ok].all() and (r.logp[~ok] == -INF).all()
            assert ((r.entropy - h).abs() <= 2e-5 * (1 + h)).all()


def test_rows_that_take_no_part_are_not_read():
    x, t = _logits(9, 2000, BF16, seed=7)
    x[2], x[5] = NAN, INF
    t[2] = t[5] = -1
    r = A.token_scores(x, t, top=2)
    assert r.logp[2] == 0 and r.entropy[5] == 0 and (r.top_ids[2] == -1).all()
    assert (r.top_logp[5] == 0).all()
    d = torch.full((9,), NAN, device="cuda")
    d[t >= 0] = 1.0
    g = A.token_scores_grad(x, t, r, d_logp=d)
    assert (g[2] == 0).all() and (g[5] == 0).all() and g.isfinite().all()


def test_ids_of_the_callers():
    """One index twice, the token among them, and what is no index."""
    x, t = _logits(2, 1000, F32, seed=10)
    r = A.token_scores(x, t, top=5)
    ids = torch.stack([t.int(), t.int(), torch.tensor([7, 999], device="cuda", dtype=torch.int32),
                       torch.full((2,), -1, device="cuda", dtype=torch.int32),
                       torch.full((2,), 1000, device="cuda", dtype=torch.int32)], 1)
    d, c = torch.tensor([0.5, -1.0], device="cuda"), torch.randn(2, 5, generator=_gen(), device="cuda")
    g = A.token_scores_grad(x, t, r._replace(top_ids=ids.contiguous()), d_logp=d, d_top=c)
    y = x.double().requires_grad_()
    lp = torch.log_softmax(y, -1)
    loss = (lp.gather(1, t[:, None])[:, 0] * d).sum() + \
        (lp.gather(1, ids[:, :3].long()) * c[:, :3]).sum()
    (want,) = torch.autograd.grad(loss, y)
    assert ((g - want).abs() <= 2e-5 * (lp.exp() * 8 + want.abs())).all()


def test_offsets_past_31_bits():
    v, rows = 65536, 32770
    x = torch.zeros(rows, v, dtype=BF16, device="cuda")
    t = torch.full((rows,), -1, device="cuda")
    x[-1] = torch.randn(v, generator=_gen(), device="cuda").to(BF16)
    t[-1] = 12345
    r = A.token_scores(x, t, top=3)
    _check(A.TokenScores(*[f[-2:] for f in r]), x[-2:], t[-2:], 3)
    want = _check_grad(x[-2:], t[-2:], 3, parts=("logp",))
    d = torch.zeros(rows, device="cuda")
    d[-2:] = torch.randn((2,), generator=_gen(5), device="cuda")
    g = A.token_scores_grad(x, t, r, d_logp=d, grad=x)
    assert torch.equal(g[-2:], want) and not g[:-2].any()


def test_reruns_streams_and_graphs():
    x, t = _logits(64, 30011, BF16, seed=12)
    d = torch.randn(64, generator=_gen(), device="cuda")

    def both(**kw):
        r = A.token_scores(x, t, top=10, **kw)
        return (*r, A.token_scores_grad(x, t, r, d_logp=d, d_entropy=d, **kw))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(stream=side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = both()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(want, other, captured):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_no_rows():
    x, t = torch.empty(0, 5, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    r = A.token_scores(x, t, top=2)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 2)
    assert A.token_scores_grad(x, t, r, d_logp=r.logp).shape == (0, 5)


def test_grad_counts_as_written():
    x, t = _logits(3, 50, F32)
    r = A.token_scores(x, t)
    before = x._version
    A.token_scores_grad(x, t, r, d_logp=r.logp, grad=x)
    assert x._version == before + 1


def test_refusals():
    x, t = _logits(3, 50, F32)
    r = A.token_scores(x, t)
    for top in (-1, 33, 51):
        with pytest.raises(ValueError):
            A.token_scores(x, t, top=top)
    with pytest.raises(ValueError):
        A.token_scores_grad(x, t, r)
    with pytest.raises(ValueError):
        A.token_scores_grad(x, t, r, d_top=torch.zeros(3, 2, device="cuda"))
    with pytest.raises(ValueError):
        A.token_scores_grad(x, t, r, d_logp=torch.zeros(4, device="cuda"))
    # rows of the logits' memory, two elements on
    base = torch.randn(152, device="cuda", generator=_gen())
    with pytest.raises(A.AlocoError):
        A.token_scores_grad(base[:-2].view(3, 50), t, r, d_logp=r.logp, grad=base[2:].view(3, 50))
