"""GPU parity of the gradient-list operators (global norm, clipping in place
and into a flat vector) against float64.

Tolerances: squares are added in fp32 over at most 32 elements (each sum off by
at most 32 u, u = 2^-24, all terms positive) and then in fp64, and the norm is
rounded to fp32: relative 17 u.  A clipped value is one product of fp32 factors,
of which the factor carries the norm's error and one rounding: 20 u, and 2^-9
more for bf16."""
import math

import numpy as np
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from paper_2609_36662_gb300 import workloads as W

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F, H = torch.float32, torch.bfloat16


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _tensors(sizes, dtypes, seed, std=1e-2, offset=0):
    """Tensors of the sizes, `offset` elements into allocations of their own."""
    out, g = [], _gen(seed)
    for i, n in enumerate(sizes):
        d = dtypes[i % len(dtypes)]
        out.append((torch.randn(n + offset, generator=g, device="cuda") * std).to(d)[offset:])
    return out


def _exact(ts):
    flat = np.concatenate([t.cpu().double().numpy().reshape(-1) for t in ts])
    return flat, float(np.sqrt(np.dot(flat, flat)))


def _assert_norm(got, want):
    got = float(got)
    if math.isnan(want):
        assert math.isnan(got)
    elif math.isinf(want) or want > 3.4e38:
        assert got == math.inf
    else:
        assert abs(got - want) <= 17 * U * want + 1e-45, (got, want)


def _assert_clipped(got, flat, norm, max_norm, dtype):
    c = min(1.0, max_norm / (norm + 1e-6))
    want = flat * c
    got = got.cpu().double().numpy().reshape(-1)
    tol = (20 * U + (2.0 ** -8 if dtype == H else 0.0)) * np.abs(want) + 1e-38
    assert got.shape == want.shape and np.all(np.abs(got - want) <= tol)


SETS = {
    "one": [1], "empty": [0], "vectors": [7, 0, 1, 4096, 33], "odd": [50257, 3, 0, 12289, 1],
    "unit": [8, 16, 24, 4, 2], "chunks": [4096, 4097, 8191, 100_003], "many": [13] * 700 + [5000],
    "large": [3_000_001, 17, 1_000_000],
}


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("dtypes", [(F,), (H,), (F, H), (H, H, F)], ids=["f", "h", "fh", "hhf"])
@pytest.mark.parametrize("name", SETS)
def test_sets(name, dtypes, offset):
    ts = _tensors(SETS[name], dtypes, 1, offset=offset)
    flat, norm = _exact(ts)
    g = A.GradList(ts)
    _assert_norm(A.grad_norm(g), norm)
    _assert_norm(A.grad_norm(ts), norm)
    max_norm = 0.3 * norm if norm > 0 else 1.0
    before = [t.clone() for t in ts]
    for od in (F, H):
        for lead in (0, 1):
            big = torch.full((len(flat) + 2 * 64 + lead,), -7.0, dtype=od, device="cuda")
            out = big[64 + lead:64 + lead + len(flat)]
            _assert_norm(A.clip_grads(g, max_norm, out=out), norm)
            _assert_clipped(out, flat, norm, max_norm, od)
            assert bool((big[:64 + lead] == -7).all()) and bool((big[64 + lead + len(flat):] == -7).all())
    assert all(torch.equal(a, b) for a, b in zip(ts, before))
    _assert_norm(A.clip_grads(g, max_norm), norm)
    at = 0
    for t in ts:
        _assert_clipped(t, flat[at:at + t.numel()], norm, max_norm, t.dtype)
        at += t.numel()


@pytest.mark.parametrize("dtype", [F, H], ids=["f32", "bf16"])
def test_below_the_threshold(dtype):
    """Nothing changes in place; the flat vector still receives everything."""
    ts = _tensors([1000, 1, 30_011], (dtype,), 2, std=1e-4)
    flat, norm = _exact(ts)
    keep = [t.clone() for t in ts]
    out = torch.full((len(flat),), -7.0, dtype=dtype, device="cuda")
    _assert_norm(A.clip_grads(ts, 1.0, out=out), norm)
    assert torch.equal(out, torch.cat(keep))
    _assert_norm(A.clip_grads(ts, 1.0), norm)
    assert all(torch.equal(a, b) for a, b in zip(ts, keep))


@pytest.mark.parametrize("dtype", [F, H], ids=["f32", "bf16"])
@pytest.mark.parametrize("v", [1e30, 3e38, 1e-30, 1e-38, 1e-44, 0.0])
def test_values_whose_squares_leave_fp32(v, dtype):
    ts = [torch.zeros(5000, dtype=dtype, device="cuda"), torch.zeros(37, dtype=dtype, device="cuda")]
    ts[0][17], ts[0][4099], ts[1][36], ts[1][0] = v, -v, v, 3 * v / 4
    flat, norm = _exact(ts)
    _assert_norm(A.grad_norm(ts), norm)
    if 0 < norm < 3e38 and norm > 1e-30:
        out = torch.empty(5037, dtype=dtype, device="cuda")
        A.clip_grads(ts, 1.0, out=out)
        _assert_clipped(out, flat, norm, 1.0, dtype)


def test_inf_and_nan():
    for bad in (math.inf, -math.inf, math.nan):
        ts = _tensors([300, 5000], (F, H), 3)
        ts[1][4000] = bad
        assert not math.isfinite(float(A.grad_norm(ts)))
        out = torch.empty(5300, device="cuda")
        norm = float(A.clip_grads(ts, 1.0, out=out))
        assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
        assert math.isnan(float(out[4300]))
        rest = torch.cat([out[:4300], out[4301:]])
        # c = 1 / inf = 0; c = NaN
        assert bool(torch.isnan(rest).all()) if math.isnan(bad) else not bool(rest.any())


def test_the_150m_set_and_the_adamw_step():
    """The 150M set's tensors, clipped into the flat vector that adamw_step
    takes: the step then equals the one that clips by itself."""
    sizes = [n for _, n, _ in W.LLAMA_150M.tensors()]
    flat = torch.randn(sum(sizes), generator=_gen(4), device="cuda") * 1e-3
    ts, at = [], 0
    for n in sizes:
        ts.append(flat[at:at + n])
        at += n
    norm = float(torch.linalg.vector_norm(flat, dtype=torch.float64))
    out = torch.empty_like(flat)
    g = A.GradList(ts)
    _assert_norm(A.grad_norm(g), norm)
    _assert_norm(A.clip_grads(g, 1.0, out=out), norm)
    state = lambda: [torch.full_like(flat, v) for v in (0.02, 1e-4, 1e-7)]
    a, b = state(), state()
    cfg = dict(lr=1e-3, step=5)
    A.adamw_step([a[0]], [out], [a[1]], [a[2]], A.adamw_cfg(max_grad_norm=0.0, **cfg))
    st = A.adamw_step([b[0]], [flat], [b[1]], [b[2]], A.adamw_cfg(max_grad_norm=1.0, **cfg))
    assert st["clip"][0] < 1.0
    for p, q in zip(a, b):
        assert torch.allclose(p, q, rtol=64 * U, atol=1e-12)


def test_a_tensor_beyond_32_bits():
    n = 2 ** 31 + 1003
    big = torch.zeros(n, dtype=H, device="cuda")
    small = torch.full((5,), 2.0, device="cuda")
    big[0], big[2 ** 31 + 7], big[n - 1] = 3.0, 4.0, 5.0
    want = math.sqrt(9 + 16 + 25 + 20)
    g = A.GradList([big, small])
    _assert_norm(A.grad_norm(g), want)
    out = torch.empty(n + 5, dtype=H, device="cuda")
    _assert_norm(A.clip_grads(g, want / 2, out=out), want)
    c = 0.5
    for at, v in ((0, 3.0), (2 ** 31 + 7, 4.0), (n - 1, 5.0), (n, 2.0), (n + 4, 2.0)):
        assert float(out[at]) == pytest.approx(c * v, rel=2.0 ** -8)
    assert float(out.abs().amax()) <= 2.51 and int(torch.count_nonzero(out)) == 8


def test_determinism_streams_and_many_calls():
    ts = _tensors([1_000_003, 77, 300_000], (H, F), 5)
    g = A.GradList(ts)
    first = A.grad_norm(g)
    out = torch.empty(g.numel, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    norms = [A.grad_norm(g, stream=side) for _ in range(20)]
    norms += [A.clip_grads(g, 1e-3, out=out, stream=side) for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, n) for n in norms)


def test_a_captured_clip_follows_its_gradients():
    ts = _tensors([40_000, 9], (F,), 6)
    g = A.GradList(ts)
    out = torch.empty(g.numel, device="cuda")
    A.clip_grads(g, 0.5, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = A.clip_grads(g, 0.5, out=out)
    for scale in (1.0, 50.0, 0.01):
        ts[0].mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        flat, want = _exact(ts)
        _assert_norm(norm, want)
        _assert_clipped(out, flat, want, 0.5, F)


def test_refusals():
    t = torch.zeros(100, device="cuda")
    for bad, err in (([], ValueError), ([t.half()], TypeError), ([t.cpu()], ValueError),
                     ([t[::2]], ValueError), ([t, t.cpu()], ValueError)):
        with pytest.raises(err):
            A.GradList(bad)
    g = A.GradList([t])
    for v in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(A.AlocoError) as e:
            A.clip_grads(g, v)
        assert e.value.status == A.ERR_ARG
    for out in (torch.zeros(99, device="cuda"), torch.zeros(100), torch.zeros(200, device="cuda")[::2]):
        with pytest.raises(ValueError):
            A.clip_grads(g, 1.0, out=out)
    with pytest.raises(TypeError):
        A.clip_grads(g, 1.0, out=torch.zeros(100, device="cuda", dtype=torch.float64))
    with pytest.raises(A.AlocoError) as e:
        A.clip_grads(g, 1.0, out=t)
    assert e.value.status == A.ERR_ALIAS
    twice = A.GradList([t, t[50:]])
    with pytest.raises(A.AlocoError) as e:
        A.clip_grads(twice, 1.0)
    assert e.value.status == A.ERR_ALIAS
    t.fill_(2.0)
    _assert_norm(A.grad_norm(twice), math.sqrt(600.0))  # reading it is fine
    t.data = torch.ones(100, device="cuda")
    with pytest.raises(ValueError):
        A.grad_norm(g)
