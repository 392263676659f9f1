"""The orthogonalised step of many replicas against the formula in 64 bits."""
import math

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from _orthogonal import allowed, momentum_like

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ODD = [(5, 100, 33), (3400, 26, 105), (6200, 50, 50), (8705, 1, 129), (8840, 77, 1), (9000, 7, 409)]
ODD_SIZE = 9000 + 7 * 409 + 3


def _state(parts, n, M, pdt, gdt, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)

    def vector(std):
        return torch.randn(n, generator=gen, device="cuda") * std

    xs = [vector(0.02).to(pdt) for _ in range(M)]
    gs, bs = [vector(1e-3) for _ in range(M)], [vector(1e-3) for _ in range(M)]
    for g, b in zip(gs, bs):
        for at, r, c in parts:
            b[at:at + r * c] = 4 * momentum_like(r, c, gen).reshape(-1)
            g[at:at + r * c] = momentum_like(r, c, gen).reshape(-1)
    return xs, [g.to(gdt) for g in gs], bs


def _scale(kind, r, c):
    return {A.MUON_ADAMW: 0.2 * math.sqrt(max(r, c)), A.MUON_ASPECT: math.sqrt(max(1, r / c)),
            A.MUON_UNIT: 1.0}[kind]


def _check(before, after, parts, lr=2e-3, mu=0.95, wd=0.1, nesterov=True, kind=A.MUON_ADAMW,
           eps=1e-7, workers=None, two_at_a_time=False):
    half = torch.finfo(after[0][0].dtype).eps / 2
    for m in workers or range(len(after[0])):
        x, g, b = (s[m] for s in before)
        x1, g1, b1 = (s[m] for s in after)
        assert torch.equal(g1, g)
        free = torch.ones(x.numel(), dtype=torch.bool, device="cuda")
        for at, r, c in parts:
            cut = slice(at, at + r * c)
            free[cut] = False
            gd, bd = g[cut].double(), b[cut].double()
            want = mu * bd + gd
            # one rounding of the sum, one of mu
            tol = 2.0 ** -24 * (want.abs() + (mu * bd).abs())
            assert ((b1[cut].double() - want).abs() <= tol + 1e-44).all()
            u = gd + mu * want if nesterov else want
            o, off = allowed(u.view(r, c), eps=eps, two_at_a_time=two_at_a_time)
            step = lr * _scale(kind, r, c)
            theta = (1 - lr * wd) * x[cut].double() - step * o.reshape(-1)
            # the factor's error, u's roundings (3 in fp32, which the steps raise
            # by no more than 3.4445^5), three roundings of the step and the store's
            tol = step * (off + 3 * 2.0 ** -24 * 485 * float(o.norm())) + \
                (half + 3 * 2.0 ** -24) * float(theta.norm())
            err = float((x1[cut].double() - theta).norm())
            assert err <= tol, (m, r, c, err, tol)
        assert torch.equal(x1[free], x[free]) and torch.equal(b1[free], b[free])


def _clone(s):
    return tuple([t.clone() for t in ts] for ts in s)


@pytest.mark.parametrize("M", [1, 3, 32])
@pytest.mark.parametrize("pdt,gdt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)],
                         ids=["f32-f32", "f32-bf16", "bf16-f32", "bf16-bf16"])
def test_matrices_at_odd_places(pdt, gdt, M):
    s = _state(ODD, ODD_SIZE, M, pdt, gdt)
    before = _clone(s)
    A.muon_step(*s, ODD, A.muon_cfg(lr=2e-3))
    _check(before, s, ODD, workers={0, M - 1})


@pytest.mark.parametrize("pdt", [F32, BF16], ids=["f32", "bf16"])
def test_layers(pdt):
    parts, at = [], 0
    for r, c in [(512, 512), (512, 64), (64, 512), (1400, 512), (512, 1400)] * 2:
        parts.append((at, r, c))
        at += r * c
    s = _state(parts, at, 2, pdt, pdt)
    before = _clone(s)
    A.muon_step(*s, A.Matrices(parts), A.muon_cfg(lr=2e-3))
    _check(before, s, parts)


@pytest.mark.parametrize("kw", [dict(nesterov=0), dict(momentum=0.0), dict(weight_decay=0.0),
                                dict(scale=A.MUON_ASPECT), dict(scale=A.MUON_UNIT), dict(lr=0.0)],
                         ids=lambda k: "-".join(k))
def test_settings(kw):
    s = _state(ODD, ODD_SIZE, 2, F32, F32, seed=1)
    before = _clone(s)
    kw = {"lr": 2e-3} | kw
    A.muon_step(*s, ODD, A.muon_cfg(**kw))
    _check(before, s, ODD, lr=kw["lr"], mu=kw.get("momentum", 0.95), wd=kw.get("weight_decay", 0.1),
           nesterov=kw.get("nesterov", 1), kind=kw.get("scale", A.MUON_ADAMW))


def test_many_shapes_and_many_matrices():
    """More shapes than one pass takes, and more matrices of a shape than its
    table of places holds."""
    gen = torch.Generator().manual_seed(2)
    parts, at = [], 1
    for _ in range(40):
        r, c = (int(v) for v in torch.randint(1, 60, (2,), generator=gen))
        parts.append((at, r, c))
        at += r * c + 3
    for _ in range(1300):
        parts.append((at, 4, 6))
        at += 25
    s = _state(parts, at, 1, F32, F32)
    before = _clone(s)
    A.muon_step(*s, parts, A.muon_cfg(lr=2e-3))
    _check_some(before, s, parts)


def _check_some(before, after, parts):
    some = parts[:40] + parts[40::97] + parts[-1:]
    for at, r, c in some:
        cut = slice(at, at + r * c)
        _check(tuple([t[cut] for t in ts] for ts in before),
               tuple([t[cut] for t in ts] for ts in after), [(0, r, c)])


@pytest.mark.parametrize("pdt", [F32, BF16], ids=["f32", "bf16"])
def test_many_wide_matrices_beside_other_shapes(pdt):
    """Two shapes of which there are many (in bf16 they take two steps at a time), and
    a few others."""
    parts, at = [], 0
    for r, c in [(300, 520)] * 30 + [(520, 256)] * 30 + [(140, 150), (9, 700), (700, 131)]:
        parts.append((at, r, c))
        at += r * c
    s = _state(parts, at, 8, pdt, BF16, seed=9)
    before = _clone(s)
    A.muon_step(*s, parts, A.muon_cfg(lr=2e-3))
    some = [parts[i] for i in (0, 17, 29, 30, 44, 59, 60, 61, 62)]
    for m in (0, 3, 7):
        for p in some:
            cut = slice(p[0], p[0] + p[1] * p[2])
            _check(tuple([ts[m][cut]] for ts in before), tuple([ts[m][cut]] for ts in s),
                   [(0, p[1], p[2])], two_at_a_time=pdt is BF16 and p in parts[:60])


def test_order_of_the_matrices_does_not_matter():
    s = _state(ODD, ODD_SIZE, 2, F32, F32)
    other = _clone(s)
    A.muon_step(*s, ODD, A.muon_cfg())
    A.muon_step(*other, ODD[::-1], A.muon_cfg())
    for a, b in zip(s, other):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_steps_follow_one_another_also_from_a_graph():
    parts = [(0, 96, 64), (96 * 64 + 1, 33, 70)]
    n = 96 * 64 + 33 * 70 + 1
    cfg = A.muon_cfg(lr=1e-2)
    eager = _state(parts, n, 2, F32, BF16)
    replayed = _clone(eager)
    for _ in range(3):
        A.muon_step(*eager, parts, cfg)
    matrices = A.Matrices(parts)
    kept = _clone(replayed)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.muon_step(*replayed, matrices, cfg)
    for a, b in zip(kept, replayed):
        for p, q in zip(a, b):
            q.copy_(p)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager, replayed):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_streams_do_not_share_scratch():
    parts = [(0, 700, 500)]
    cfg = A.muon_cfg(lr=1e-2)
    a, b = (_state(parts, 350000, 1, F32, F32, seed=i) for i in (3, 4))
    want = [_clone(a), _clone(b)]
    for s in want:
        for _ in range(4):
            A.muon_step(*s, parts, cfg)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, st in zip((a, b), streams):
            A.muon_step(*s, parts, cfg, stream=st)
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        assert all(torch.equal(p, q) for p, q in zip(s[0] + s[2], w[0] + w[2]))


def test_nan_stays_in_its_matrix():
    s = _state(ODD, ODD_SIZE, 2, F32, F32)
    clean = _clone(s)
    s[1][1][ODD[1][0] + 3] = float("nan")
    A.muon_step(*s, ODD, A.muon_cfg())
    A.muon_step(*clean, ODD, A.muon_cfg())
    at, r, c = ODD[1]
    assert s[0][1][at:at + r * c].isnan().all()
    s[0][1][at:at + r * c] = clean[0][1][at:at + r * c]
    assert torch.equal(s[0][1], clean[0][1]) and torch.equal(s[0][0], clean[0][0])


def test_offsets_past_31_bits():
    """A matrix behind more than 2^31 elements of a bf16 replica."""
    n, at = (1 << 31) + 70 * 40 + 9, (1 << 31) + 7
    x, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    b = torch.zeros(n, device="cuda")
    gen = torch.Generator("cuda").manual_seed(5)
    x[at:at + 2800] = torch.randn(2800, generator=gen, device="cuda").to(BF16) * 0.02
    g[at:at + 2800] = momentum_like(70, 40, gen).reshape(-1).to(BF16)
    tail = [([t[at - 7:].clone()]) for t in (x, g, b)]
    A.muon_step([x], [g], [b], [(at, 70, 40)], A.muon_cfg(lr=2e-3))
    assert not x[:at].any() and not b[:at].any()
    _check(tail, [[t[at - 7:]] for t in (x, g, b)], [(7, 70, 40)])


def test_no_matrices():
    s = _state([], 10, 1, F32, F32)
    before = _clone(s)
    A.muon_step(*s, [], A.muon_cfg())
    A.muon_step(*s, [(3, 0, 5), (10, 4, 0)], A.muon_cfg())
    assert all(torch.equal(p[0], q[0]) for p, q in zip(s, before))


def test_what_a_step_writes_counts_as_written():
    s = _state([(0, 8, 8)], 64, 1, F32, F32)
    versions = [t._version for t in (s[0][0], s[2][0])]
    A.muon_step(*s, [(0, 8, 8)], A.muon_cfg())
    assert [t._version for t in (s[0][0], s[2][0])] == [v + 1 for v in versions]
