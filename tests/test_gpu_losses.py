"""GPU parity of the post-training losses (token log-probabilities, policy and
preference loss with their gradients by the logits) against float64, at the
sizes, layouts and masks where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import _losses as L
from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

BOTH = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]
# one element, below and above a 16-byte unit, a block's and a cluster's ends,
# the repository's vocabularies, odd ones, the largest
VOCABS = [1, 2, 7, 8, 9, 33, 257, 1000, 4087, 4088, 4089, 8191, 16384, 16385, 32000, 50257,
          128256, 131065, 131072, A.MAX_VOCAB]
LO, HI, KL = 0.2, 0.28, 0.04


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _logits(shape, dtype, seed, std=2.0):
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * std).to(dtype)


def _targets(shape, V, seed, dtype=torch.int64):
    return torch.randint(0, V, shape, generator=_gen(seed + 1), device="cuda").to(dtype)


def _h(t):
    return t.detach().cpu().double().numpy()


def _flat(x):
    return _h(x).reshape(-1, x.shape[-1])


def _policy_inputs(x, t, tau, seed, masked=True):
    """Advantages, old and reference log-probabilities near the logits' own, no
    ratio at an edge of the clipping range, and weights with zeros."""
    rng = np.random.default_rng(seed)
    with np.errstate(all="ignore"):
        lp, _ = L.logprobs(_flat(x), np.clip(_h(t).astype(np.int64).reshape(-1), 0, x.shape[-1] - 1),
                           tau)
    lp = np.nan_to_num(lp, nan=-1.0, posinf=0.0, neginf=-20.0)
    n = lp.size
    old = (lp + rng.normal(0, 0.25, n)).astype(np.float32)
    for edge in (1 - LO, 1 + HI):
        old += np.where(np.abs(np.exp(lp - old) - edge) < 5e-3, np.float32(0.03), np.float32(0))
    w = rng.uniform(0.2, 1.0, n)
    if masked and n > 2:
        w[::3] = 0.0
    w /= max(w.sum(), 1e-9)
    a = dict(adv=rng.normal(0, 1, n), old=old, w=w, ref=lp + rng.normal(0, 0.3, n))
    return {k: torch.tensor(v, dtype=torch.float32, device="cuda").reshape(t.shape)
            for k, v in a.items()}


def _check_policy(x, t, a, tau, got, x0=None, kl=KL):
    """Compare a PolicyLoss with float64 on the same inputs (x0: the logits
    before the call, where it wrote over them)."""
    th = _h(t).astype(np.int64).reshape(-1)
    ref = a.get("ref")
    o = L.policy(_flat(x0 if x0 is not None else x), th, _h(a["adv"]).reshape(-1),
                 _h(a["old"]).reshape(-1), _h(a["w"]).reshape(-1),
                 _h(ref).reshape(-1) if ref is not None else None, LO, HI, kl, tau)
    L.assert_logp(_h(got.logp), o["logp"], x.shape[-1], o["live"])
    L.assert_terms(_h(got.terms), o)
    if got.grad is not None:
        L.assert_grad(_flat(got.grad), o, th, x.dtype == torch.bfloat16)
    return o


def _policy(x, t, a, tau=1.0, kl=KL, **kw):
    return A.policy_loss(x, t, a["adv"], a["old"], a["w"], ref_logp=a.get("ref"), clip_low=LO,
                         clip_high=HI, kl_coef=kl, temperature=tau, **kw)


# ------------------------------------------------------------- vocabularies

@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("V", VOCABS)
def test_every_vocabulary(V, dtype):
    """Five contiguous rows: for odd vocabularies every phase of a row to the
    16-byte boundaries occurs."""
    x, t = _logits((5, V), dtype, V), _targets((5,), V, V)
    t[3] = -7
    lp, _ = L.logprobs(_flat(x), _h(t).astype(np.int64), 1.0)
    L.assert_logp(_h(A.token_logprobs(x, t)), lp, V)
    a = _policy_inputs(x, t, 1.0, V)
    _check_policy(x, t, a, 1.0, _policy(x, t, a))
    _check_preference(x, t, [0, 2, 5], a["ref"], 1.0)


def _check_preference(x, t, cu, ref, tau, beta=0.1, eps=0.05, x0=None, **kw):
    cu_t = cu if torch.is_tensor(cu) else torch.tensor(cu, dtype=torch.int32, device="cuda")
    th = _h(t).astype(np.int64).reshape(-1)
    o = L.preference(_flat(x0 if x0 is not None else x), th, cu_t.cpu().numpy(),
                     _h(ref).reshape(-1) if ref is not None else None, beta, eps, tau)
    got = A.preference_loss(x, t, cu_t, ref, beta=beta, label_smoothing=eps, temperature=tau, **kw)
    L.assert_logp(_h(got.logp), o["logp"], x.shape[-1], o["live"])
    L.assert_preference(_h(got.loss), _h(got.log_ratios), o, cu_t.cpu().numpy(), beta, x.shape[-1])
    if got.grad is not None:
        L.assert_grad(_flat(got.grad), o, th, x.dtype == torch.bfloat16)
    return got


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("rows,V", [(1, 50257), (2, 700), (3, 32000), (700, 260), (400, 4500),
                                    (331, 12001), (160, 32000)])
def test_row_counts(rows, V, dtype):
    """One row (the vocabulary is split over SMs) to several rows an SM."""
    x, t = _logits((rows, V), dtype, rows), _targets((rows,), V, rows, torch.int32)
    a = _policy_inputs(x, t, 0.7, rows)
    o = _check_policy(x, t, a, 0.7, _policy(x, t, a, 0.7))
    L.assert_logp(_h(A.token_logprobs(x, t, temperature=0.7)),
                  L.logprobs(_flat(x), _h(t).astype(np.int64), 0.7)[0], V)
    assert o["live"].any()
    cu = [0, rows // 3, rows - rows // 4]
    _check_preference(x, t, cu, a["ref"], 0.7)


@pytest.mark.parametrize("dtype,rows,V", [(torch.float32, 1400, 16000), (torch.bfloat16, 2700, 16001)],
                         ids=IDS)
def test_calls_whose_sums_take_a_kernel_of_their_own(dtype, rows, V):
    """Over 80 MB of logits the policy loss's sums are a second kernel's."""
    x, t = _logits((rows, V), dtype, 3), _targets((rows,), V, 3)
    a = _policy_inputs(x, t, 1.0, 3)
    _check_policy(x, t, a, 1.0, _policy(x, t, a))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("rows,pairs", [(3000, 40), (2500, 1), (60, 30), (2049, 2)])
def test_many_rows_and_many_pairs(rows, pairs, dtype):
    """More rows or pairs than one block of the row kernel works out by itself;
    ragged sequences, some of them empty."""
    x, t = _logits((rows, 257), dtype, rows), _targets((rows,), 257, rows)
    t[::5] = -1
    rng = np.random.default_rng(rows + pairs)
    cu = np.sort(rng.integers(0, rows + 1, 2 * pairs + 1))
    ref = torch.randn(rows, generator=_gen(pairs), device="cuda") - 5.0
    _check_preference(x, t, torch.tensor(cu, device="cuda"), ref, 1.0)
    _check_preference(x, t, torch.tensor(cu, device="cuda"), ref, 1.0, want_grad=False)


# -------------------------------------------------------------------- layouts

@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("V", [33, 5001, 32000])
@pytest.mark.parametrize("how", ["shifted", "by_position", "padded", "offset", "in_place"])
def test_layouts(how, V, dtype):
    """Views without each sequence's last position, sequence-last layouts,
    padded rows, a start off every boundary, the gradient over the logits."""
    B, T = 3, 4
    pad = 0
    if how == "shifted":
        x = _logits((B, T + 1, V), dtype, 1)[:, :T]
    elif how == "by_position":
        x = _logits((T, B, V), dtype, 2).transpose(0, 1)
    elif how == "padded":
        pad = 13
        x = _logits((B, T, V + pad), dtype, 3)[..., :V]
    elif how == "offset":
        x = _logits((B * T * V + 3,), dtype, 4)[3:].view(B, T, V)
    else:
        x = _logits((B, T, V), dtype, 5)
    t = _targets((B, T), V, 6)
    t[1, 2] = -1
    a = _policy_inputs(x, t, 1.0, 7)
    x0 = x.clone()
    kw = {"grad": x} if how == "in_place" else {}
    got = _policy(x, t, a, **kw)
    _check_policy(x, t, a, 1.0, got, x0)
    if how == "in_place":
        assert got.grad.data_ptr() == x.data_ptr()
        x.copy_(x0)
        kw["grad"] = x
    else:
        assert torch.equal(x, x0)
    _check_preference(x, t, [0, 3, 5, 9, 12], a["ref"], 1.0, x0=x0, **kw)
    if how != "in_place":
        assert torch.equal(x, x0)


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("xo,go,V", [(0, 1, 4001), (1, 0, 4001), (3, 2, 32001), (0, 5, 130),
                                     (2, 2, 40000)])
def test_gradient_of_another_phase_stays_within_its_rows(xo, go, V, dtype):
    """Logits and gradient rows that lie differently to the 16-byte boundaries;
    what lies between and around the gradient's rows is not written."""
    n, pad = 4, 17
    xb = torch.full((n * (V + pad) + xo,), 3.0, dtype=dtype, device="cuda")
    x = xb[xo:].view(n, V + pad)[:, :V]
    x.copy_(_logits((n, V), dtype, V))
    gb = torch.full((n * (V + pad) + go,), -7.0, dtype=dtype, device="cuda")
    g = gb[go:].view(n, V + pad)[:, :V]
    t = _targets((n,), V, V)
    a = _policy_inputs(x, t, 1.0, V, masked=False)
    a["w"][2] = 0.0
    _check_policy(x, t, a, 1.0, _policy(x, t, a, grad=g))
    rest = gb[go:].view(n, V + pad)[:, V:]
    assert bool((rest == -7.0).all()) and bool((gb[:go] == -7.0).all())
    g.fill_(1.0)
    _check_preference(x, t, [0, 2, 4], a["ref"], 1.0, grad=g)
    assert bool((rest == -7.0).all()) and bool((gb[:go] == -7.0).all())


def test_rows_beyond_32_bits_of_elements():
    V, stride = 32001, 2 ** 31 + 8
    buf = torch.empty(stride + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, V), (stride, 1))
    x.copy_(_logits((2, V), torch.bfloat16, 3))
    t = _targets((2,), V, 4)
    a = _policy_inputs(x, t, 1.0, 5, masked=False)
    x0 = x.clone()
    _check_policy(x, t, a, 1.0, _policy(x, t, a, grad=x), x0)
    x.copy_(x0)
    _check_preference(x, t, [0, 1, 2], a["ref"], 1.0, x0=x0, grad=x)


# ---------------------------------------------------------------- rows, masks

@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("V", [40, 9001, 50000])
def test_special_values(V, dtype):
    """Banned tokens (-inf, the type's lowest value), rows of the lowest value,
    of nothing but -inf, with NaN and with +inf, a banned token asked for, a
    token beyond the vocabulary, and NaN in rows that take no part."""
    low = torch.finfo(dtype).min
    x, t = _logits((12, V), dtype, V), _targets((12,), V, V)
    x[0, 1::2] = -math.inf
    t[0] = 0
    x[1, 3:] = low
    t[1] = 2
    x[2, :] = low
    x[3, :] = -math.inf
    x[4, V // 2] = math.nan
    x[5, V // 3] = math.inf
    x[6, 5] = -math.inf
    t[6] = 5
    t[7] = V
    x[8, :] = math.nan           # weight 0
    t[9] = -100
    x[9, :] = math.nan           # no token
    x[10, :] = -3e38 if dtype == torch.float32 else -3.0e38
    x[10, V - 1] = 3e38          # the difference leaves the range
    t[10] = V - 1
    x[11, :] = -1000.0
    a = _policy_inputs(x, t, 1.0, V, masked=False)
    a["w"][8] = 0.0
    got = _policy(x, t, a)
    o = _check_policy(x, t, a, 1.0, got)
    for row in (3, 4, 5, 7):
        assert math.isnan(float(got.logp[row]))
    assert float(got.logp[6]) == -math.inf
    assert float(got.logp[10]) == 0.0
    assert not bool(got.grad[8].any()) and not bool(got.grad[9].any())
    assert abs(float(got.logp[2]) + math.log(V)) < 1e-5
    t[8] = -1
    live = [0, 1, 2, 8, 9, 10, 11]  # a pair of finite rows and rows left out
    xs, ts, ref = x[live].contiguous(), t[live].contiguous(), a["ref"][live].contiguous()
    _check_preference(xs, ts, [0, 3, 7], ref, 1.0)
    # NaN in one pair leaves the other pair's gradient alone
    pair = A.preference_loss(x, t, torch.tensor([0, 1, 3, 4, 5], device="cuda"), a["ref"])
    assert bool(torch.isfinite(pair.grad[:3]).all()) and bool(torch.isnan(pair.grad[4]).all())
    assert math.isnan(float(pair.loss)) and bool(torch.isfinite(pair.log_ratios[:2]).all())
    assert o["live"].sum() == 10


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_rows_that_all_take_no_part(dtype):
    V = 5000
    x = torch.full((4, V), math.nan, dtype=dtype, device="cuda")
    t = torch.full((4,), -1, dtype=torch.int64, device="cuda")
    z = torch.zeros(4, device="cuda")
    nan = torch.full((4,), math.nan, device="cuda")
    assert not bool(A.token_logprobs(x, t).any())
    for tt, w in ((t, z + 1), (t + 1, z)):
        got = A.policy_loss(x, tt, nan, nan, w, ref_logp=nan, kl_coef=0.1)
        assert not bool(got.terms.any()) and not bool(got.logp.any())
        assert not bool(got.grad.any())
    got = A.preference_loss(x, t, torch.tensor([0, 2, 4], device="cuda"), nan)
    assert float(got.loss) == pytest.approx(math.log(2), rel=1e-6)
    assert not bool(got.log_ratios.any()) and not bool(got.grad.any())


def test_no_rows_and_no_pairs():
    for dtype in BOTH:
        x = torch.empty(0, 100, dtype=dtype, device="cuda")
        t = torch.empty(0, dtype=torch.int64, device="cuda")
        f = torch.empty(0, device="cuda")
        assert A.token_logprobs(x, t).shape == (0,)
        got = A.policy_loss(x, t, f, f, f)
        assert not bool(got.terms.any()) and got.grad.shape == (0, 100)
        none = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = A.preference_loss(x, t, none)
        assert float(got.loss) == 0.0 and got.log_ratios.numel() == 0
        one = torch.zeros(3, dtype=torch.int32, device="cuda")
        assert float(A.preference_loss(x, t, one).loss) == pytest.approx(math.log(2), rel=1e-6)
        x = _logits((3, 100), dtype, 1)
        t = _targets((3,), 100, 1)
        assert not bool(A.preference_loss(x, t, none).grad.any())


def test_bounds_outside_the_rows_and_rows_of_no_sequence():
    V = 3001
    x, t = _logits((9, V), torch.float32, 8), _targets((9,), V, 8)
    for dt in (torch.int32, torch.int64):
        cu = torch.tensor([-5, 2, 4, 4, 300], dtype=dt, device="cuda")
        _check_preference(x, t, cu, None, 1.0)
        cu = torch.tensor([2, 3, 5], dtype=dt, device="cuda")
        got = _check_preference(x, t, cu, None, 1.0, eps=0.0)
        assert not bool(got.grad[:2].any()) and not bool(got.grad[5:].any())
        assert bool(got.grad[2:5].any(-1).all())


@pytest.mark.parametrize("scale", [1e-3, 1.0, 300.0])
def test_margins_far_from_zero(scale):
    """Large log ratios on either side: no overflow in the loss or its slope."""
    V = 500
    x, t = _logits((8, V), torch.float32, 9), _targets((8,), V, 9)
    ref = torch.tensor([scale, 0, 0, -scale, -scale, 0, 0, scale], device="cuda") - 6.0
    _check_preference(x, t, [0, 2, 4, 6, 8], ref, 1.0, beta=0.5, eps=0.0)
    _check_preference(x, t, [0, 2, 4, 6, 8], ref, 1.0, beta=0.5, eps=0.3)


def test_policy_without_reference_and_with_extreme_ratios():
    V = 2000
    x, t = _logits((6, V), torch.float32, 10), _targets((6,), V, 10)
    a = _policy_inputs(x, t, 1.0, 10, masked=False)
    del a["ref"]
    got = _policy(x, t, a, kl=0.0)
    _check_policy(x, t, a, 1.0, got, kl=0.0)
    assert float(got.terms[2]) == 0.0
    # a ratio of exp(80) with a positive advantage is clipped: no gradient; with
    # a negative one it counts in full
    a["old"][:2] -= 80.0
    a["adv"][0], a["adv"][1] = 1.0, -1.0
    got = _policy(x, t, a, kl=0.0)
    assert not bool(got.grad[0].any())
    assert float(got.grad[1].abs().max()) > 1e30
    # a negative advantage below the range is clipped, a positive one is not
    a["old"][2:4] += 81.0
    a["adv"][2], a["adv"][3] = -1.0, 1.0
    got = _policy(x, t, a, kl=0.0)
    assert not bool(got.grad[2].any()) and float(got.grad[3].abs().max()) < 1e-20


# ---------------------------------------------------------------- behaviour

@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_values_only(dtype):
    """want_grad=False gives the same terms and logp, bit for bit."""
    x, t = _logits((9, 40001), dtype, 11), _targets((9,), 40001, 11)
    a = _policy_inputs(x, t, 1.0, 11)
    with_g, without = _policy(x, t, a), _policy(x, t, a, want_grad=False)
    assert without.grad is None
    assert torch.equal(with_g.terms, without.terms) and torch.equal(with_g.logp, without.logp)
    cu = torch.tensor([0, 4, 9], device="cuda")
    with_g = A.preference_loss(x, t, cu, a["ref"])
    without = A.preference_loss(x, t, cu, a["ref"], want_grad=False)
    assert without.grad is None and torch.equal(with_g.loss, without.loss)
    assert torch.equal(with_g.log_ratios, without.log_ratios)


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("rows,V", [(200, 32000), (37, 128256), (3, 50257)])
def test_repeated_calls_are_bit_identical_and_streams_do_not_matter(rows, V, dtype):
    x, t = _logits((rows, V), dtype, 12), _targets((rows,), V, 12)
    a = _policy_inputs(x, t, 1.0, 12)
    cu = torch.tensor([0, rows // 2, rows], device="cuda")
    first = [*_policy(x, t, a), *A.preference_loss(x, t, cu, a["ref"]), A.token_logprobs(x, t)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (None, side):
        again = [*_policy(x, t, a, stream=s), *A.preference_loss(x, t, cu, a["ref"], stream=s),
                 A.token_logprobs(x, t, stream=s)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_two_streams_at_once():
    """Calls in flight on two streams, many times over, keep apart."""
    jobs = []
    for k in range(2):
        x, t = _logits((64, 30011), torch.bfloat16, 20 + k), _targets((64,), 30011, 20 + k)
        a = _policy_inputs(x, t, 1.0, 20 + k)
        cu = torch.tensor([0, 10, 30, 31, 64], device="cuda")
        want = [*_policy(x, t, a), *A.preference_loss(x, t, cu, a["ref"])]
        jobs.append((x, t, a, cu, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for k, (x, t, a, cu, _, s) in enumerate(jobs):
            got[k].append([*_policy(x, t, a, stream=s),
                           *A.preference_loss(x, t, cu, a["ref"], stream=s)])
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(p, q) for p, q in zip(g, jobs[k][4]))


def test_calls_in_a_cuda_graph():
    x, t = _logits((20, 32000), torch.bfloat16, 30), _targets((20,), 32000, 30)
    a = _policy_inputs(x, t, 1.0, 30)
    cu = torch.tensor([0, 10, 20], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _policy(x, t, a)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [*_policy(x, t, a), *A.preference_loss(x, t, cu, a["ref"])]
    for seed in (31, 32):
        x.copy_(_logits((20, 32000), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        want = [*_policy(x, t, a), *A.preference_loss(x, t, cu, a["ref"])]
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("V", [90, 4500, 20001])
def test_gradients_against_differences(V):
    """The loss's own difference along a direction.  Tolerance: the loss rounds
    to u |L| and its rows to tol_logp, over 2 h; the third derivative's term is
    h^2 times the direction's scale.  Rows whose ratio crosses an edge of the
    clipping range on the way have a kink there and take no part."""
    x, t = _logits((6, V), torch.float32, 40), _targets((6,), V, 40)
    a = _policy_inputs(x, t, 1.0, 40, masked=False)
    # along the tokens and the largest logits, where the loss moves
    D = torch.zeros_like(x)
    D.scatter_(1, t[:, None], 1.0)
    D.scatter_(1, x.topk(3).indices, -0.5)
    h = 2.0 ** -6
    th = _h(t).astype(np.int64)
    ends = [np.exp(L.logprobs(_flat(y), th, 1.0)[0] - _h(a["old"])) for y in (x - h * D, x + h * D)]
    for edge in (1 - LO, 1 + HI):
        crossed = (ends[0] < edge) != (ends[1] < edge)
        a["w"] *= torch.tensor(~crossed, device="cuda").float()
    cu = torch.tensor([0, 3, 6], device="cuda")
    calls = [lambda y: (lambda r: (r.terms[0], r.grad))(_policy(y, t, a)),
             lambda y: (lambda r: (r.loss, r.grad))(A.preference_loss(y, t, cu, a["ref"], beta=0.5))]
    for f in calls:
        diff = (float(f(x + h * D)[0]) - float(f(x - h * D)[0])) / (2 * h)
        want = float((f(x)[1].double() * D.double()).sum())
        tol = 4 * L.tol_logp(12.0, V) / (2 * h) + 4 * h * h
        assert abs(diff - want) <= tol, (diff, want, tol)


@pytest.mark.parametrize("V", [90, 4500, 40000])
def test_one_row_against_differences(V):
    """The same for single rows of weight 1, whose loss moves by about 1: the
    difference says much more there than its tolerance."""
    x, t = _logits((5, V), torch.float32, 60), _targets((5,), V, 60)
    one, h = torch.ones(1, device="cuda"), 2.0 ** -6
    tol = 4 * L.tol_logp(16.0, V) / (2 * h) + 4 * h * h
    moved = 0
    for i in range(5):
        y, a = x[i:i + 1], t[i:i + 1]
        D = torch.zeros_like(y).scatter_(1, a[:, None], 1.0).scatter_(1, y.topk(3).indices, -1.0)
        lp = A.token_logprobs(y, a)
        cu = torch.tensor([0, 1, 1] if i % 2 else [0, 0, 1], device="cuda")
        for f in (lambda z: (lambda r: (r.terms[0], r.grad))(A.policy_loss(
                      z, a, -one, lp, one, ref_logp=lp - 0.5, kl_coef=0.2)),
                  lambda z: (lambda r: (r.loss, r.grad))(A.preference_loss(z, a, cu, lp, beta=1.0))):
            diff = (float(f(y + h * D)[0]) - float(f(y - h * D)[0])) / (2 * h)
            want = float((f(y)[1].double() * D.double()).sum())
            assert abs(diff - want) <= tol, (i, diff, want, tol)
            moved += abs(want) > 30 * tol
    assert moved >= 8


# ----------------------------------------------------------------- refusals

def _args(V=64, n=4):
    x, t = _logits((n, V), torch.float32, 50), _targets((n,), V, 50)
    f = torch.zeros(n, device="cuda")
    return x, t, f


@pytest.mark.parametrize("bad,err", [
    (dict(logits="f16"), TypeError), (dict(logits="1d"), ValueError),
    (dict(logits="cols"), ValueError), (dict(logits="cpu"), ValueError),
    (dict(targets="i16"), TypeError), (dict(targets="short"), ValueError),
    (dict(targets="stride"), ValueError), (dict(adv="f64"), ValueError),
    (dict(adv="short"), ValueError), (dict(temperature=0.0), A.AlocoError),
    (dict(temperature=math.nan), A.AlocoError), (dict(clip_low=-0.1), A.AlocoError),
    (dict(clip_high=math.inf), A.AlocoError), (dict(kl_coef=0.1), A.AlocoError),
    (dict(kl_coef=-1.0), A.AlocoError), (dict(grad="bf16"), ValueError),
    (dict(grad="shape"), ValueError), (dict(grad="shifted"), A.AlocoError),
    (dict(logits="wide"), A.AlocoError), (dict(logits="overlap"), A.AlocoError),
    (dict(grad="overlap"), A.AlocoError)])
def test_refusals(bad, err):
    x, t, f = _args()
    kw = {k: v for k, v in bad.items() if k not in ("logits", "targets", "adv", "grad")}
    adv = f
    lg = bad.get("logits")
    if lg == "f16":
        x = x.half()
    elif lg == "1d":
        x, t, f = x[0], t[0], f[0]
        adv = f
    elif lg == "cols":
        x = x.t().contiguous().t()
    elif lg == "cpu":
        x = x.cpu()
    elif lg == "wide":
        x = torch.zeros(4, A.MAX_VOCAB + 1, device="cuda")
    elif lg == "overlap":
        x = x.as_strided((4, 64), (60, 1))
    tg = bad.get("targets")
    if tg == "i16":
        t = t.short()
    elif tg == "short":
        t = t[:3]
    elif tg == "stride":
        t = torch.stack([t, t], 1)[:, 0]
    if bad.get("adv") == "f64":
        adv = f.double()
    elif bad.get("adv") == "short":
        adv = f[:2]
    gr = bad.get("grad")
    if gr == "bf16":
        kw["grad"] = torch.empty_like(x, dtype=torch.bfloat16)
    elif gr == "shape":
        kw["grad"] = torch.empty(4, 65, device="cuda")
    elif gr == "shifted":  # over the logits, but not at their place
        buf = torch.zeros(4 * 64 + 4, device="cuda")
        x, kw["grad"] = buf[:256].view(4, 64), buf[4:].view(4, 64)
    elif gr == "overlap":
        kw["grad"] = torch.zeros(4 * 64, device="cuda").as_strided((4, 64), (32, 1))
    with pytest.raises(err):
        A.policy_loss(x, t, adv, f, f, **kw)


def test_preference_refusals():
    x, t, f = _args()
    cu = torch.tensor([0, 2, 4], device="cuda")
    for kw, err in ((dict(beta=0.0), A.AlocoError), (dict(beta=math.nan), A.AlocoError),
                    (dict(label_smoothing=1.0), A.AlocoError),
                    (dict(label_smoothing=-0.1), A.AlocoError)):
        with pytest.raises(err):
            A.preference_loss(x, t, cu, f, **kw)
    for c, err in ((cu[:2], ValueError), (cu.float(), TypeError), (cu.cpu(), ValueError),
                   (cu[None], ValueError)):
        with pytest.raises(err):
            A.preference_loss(x, t, c, f)
    with pytest.raises(ValueError):
        A.preference_loss(x, t, cu, f[:2])
    # what was refused left nothing behind
    assert math.isfinite(float(A.preference_loss(x, t, cu, f).loss))
