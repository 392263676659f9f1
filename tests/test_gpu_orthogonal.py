"""Orthogonal factors of matrices against the steps in 64 bits."""
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from _orthogonal import COEFFICIENTS, allowed, exact, momentum_like

pytestmark = pytest.mark.gpu


def _gen(seed=0):
    return torch.Generator("cuda").manual_seed(seed)


def _check(x, out, **kw):
    """bf16 rounds once more: half a step, relative to the value."""
    e, tol = allowed(x, **kw)
    tol += torch.finfo(torch.bfloat16).eps / 2 * float(e.norm())
    got = out.double()
    assert torch.isfinite(got).all()
    assert float((got - e).norm()) <= tol, (float((got - e).norm()), tol)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 2), (5, 3), (16, 16), (31, 33), (63, 65), (64, 64), (127, 129),
          (128, 128), (129, 127), (200, 72), (72, 200), (255, 257), (256, 256), (257, 513),
          (300, 1025), (1025, 300), (384, 384), (640, 641), (1, 5000), (5000, 1), (3, 4099),
          (2048, 16), (17, 9001), (1030, 1030),
          (128, 2049), (4096, 128), (100, 4097), (33, 511), (300, 31), (2000, 127), (129, 4096)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_matrices_of_many_shapes(shape, dtype):
    x = momentum_like(*shape, _gen()).to(dtype)
    _check(x, A.orthogonalize(x))


@pytest.mark.parametrize("shape", [(40, 768, 768), (300, 64, 130), (5, 300, 200), (3, 1, 1),
                                   (7, 200, 1024), (700, 8, 8), (700, 200, 256), (2, 400, 6000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_batches(shape):
    """The first, some and the last matrix of a batch."""
    x = torch.stack([momentum_like(*shape[1:], _gen(i)) for i in range(shape[0])])
    out = A.orthogonalize(x)
    for i in {0, 1, shape[0] // 2, shape[0] - 1}:
        _check(x[i], out[i])
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("steps", [1, 2, 3, 5])
@pytest.mark.parametrize("shape", [(260, 129, 500), (60, 300, 520), (52, 700, 260)],
                         ids=lambda s: "x".join(map(str, s)))
def test_wide_matrices_that_take_two_steps_at_a_time(shape, steps):
    x = torch.stack([momentum_like(*shape[1:], _gen(i)) for i in range(shape[0])])
    x[7] = torch.randn(shape[1:], generator=_gen(50), device="cuda")
    x[9] = 0
    x[11, 5, 5] = float("nan")
    out = A.orthogonalize(x, coefficients=[COEFFICIENTS] * steps)
    for i in (0, 7, 8, shape[0] - 1):
        _check(x[i], out[i], steps=steps, two_at_a_time=True)
    assert (out[9] == 0).all() and out[11].isnan().all()
    mixed = [(3.9, -6.2, 2.6), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)][:steps]
    out = A.orthogonalize(x, coefficients=mixed)
    _check(x[8], out[8], coefficients=mixed, two_at_a_time=True)


@pytest.mark.parametrize("kind", ["square", "wide", "rank_one", "decaying", "equal", "large",
                                  "small", "sparse"])
def test_kinds_of_spectra(kind):
    g = _gen(3)
    x = torch.randn(320, 320 if kind == "square" else 700, generator=g, device="cuda")
    if kind == "rank_one":
        x = x[:, :1] @ x[:1]
    elif kind == "decaying":
        u, _, v = torch.linalg.svd(x.double(), full_matrices=False)
        x = ((u * torch.logspace(0, -4, 320, dtype=torch.float64, device="cuda")) @ v).float()
    elif kind == "equal":
        x = torch.linalg.qr(x.T.double())[0].T.float().contiguous()
    elif kind == "large":
        x = x * 1e30
    elif kind == "small":
        x = x * 1e-25
    elif kind == "sparse":
        x = x * (torch.rand(x.shape, generator=g, device="cuda") < 0.002)
    eps = 1e-30 if kind == "small" else 1e-7
    _check(x, A.orthogonalize(x, eps=eps), eps=eps)


def test_views():
    """Padded rows, every other matrix of a batch, starts off any boundary."""
    base = momentum_like(6 * 150, 260, _gen(4)).view(6, 150, 260)
    for x in (base[:, :133, 1:202], base[::2, 5:, 3:], base[1, :, 7:100], base[:, 40:41, :],
              base.transpose(0, 1)[:7, :, 8:], base[2].expand(3, -1, -1)):
        out = A.orthogonalize(x)
        assert out.shape == x.shape and out.is_contiguous()
        for i in ([0, x.shape[0] - 1] if x.dim() == 3 else [None]):
            _check(x if i is None else x[i], out if i is None else out[i])


def test_coefficients_of_every_step():
    steps = [(3.9, -6.2, 2.6), (2.8, -3.9, 1.6), (1.875, -1.25, 0.375)]
    x = momentum_like(150, 333, _gen(5))
    _check(x, A.orthogonalize(x, coefficients=steps), coefficients=steps)
    one = A.orthogonalize(x, coefficients=[COEFFICIENTS])
    _check(x, one, steps=1)
    many = [(1.5, -0.5, 0.0)] * 16
    _check(x, A.orthogonalize(x, coefficients=many), coefficients=many)


@pytest.mark.parametrize("shape", [(3, 40, 200), (2, 140, 300), (60, 300, 520)],
                         ids=["small", "tiles", "two_steps"])
def test_polynomials_without_products(shape):
    """b = c = 0: X times the steps' a.  Rounded to bf16 once; X before that to 22
    bits, or 2^-33 where fp16's least value counts."""
    x = torch.randn(shape, generator=_gen(6), device="cuda")
    out = A.orthogonalize(x, coefficients=[[1.7, 0, 0], [0.6, 0.0, 0.0]])
    want = 1.7 * 0.6 * x.double() / (x.double().square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    assert ((out.double() - want).abs() <= (2.0**-8 + 2.0**-19) * want.abs() + 2.0**-31).all()


@pytest.mark.parametrize("eps", [3.0, 1e20, 1e39, 1e300])
@pytest.mark.parametrize("shape", [(40, 200), (140, 300)], ids=["small", "tiles"])
def test_eps_of_any_size(shape, eps):
    x = torch.randn(shape, generator=_gen(7), device="cuda")
    out = A.orthogonalize(x, eps=eps)
    if eps == 3.0:
        _check(x, out, eps=eps)
    else:
        # 3.4445^5 |x| / eps < 485 * 6 / 1e20, or nothing where X is fp16 values
        assert (out.abs() < 1e-16).all()


def test_coefficients_in_any_sequence():
    x = momentum_like(40, 60, _gen(8))
    first = A.orthogonalize(x)
    for c in ([list(COEFFICIENTS)] * 5, (list(COEFFICIENTS),) * 5, iter([COEFFICIENTS] * 5)):
        assert torch.equal(A.orthogonalize(x, coefficients=c), first)


def test_zeros_and_what_is_not_finite():
    x = torch.stack([momentum_like(130, 150, _gen(i)) for i in range(5)])
    alone = A.orthogonalize(x)
    x[1] = 0
    x[2, 7, 9] = float("nan")
    x[3, 129, 149] = float("inf")
    out = A.orthogonalize(x)
    assert (out[1] == 0).all()
    assert out[2].isnan().all() and out[3].isnan().all()
    assert torch.equal(out[0], alone[0]) and torch.equal(out[4], alone[4])


def test_reruns_streams_and_out():
    x = torch.stack([momentum_like(400, 520, _gen(i)) for i in range(6)])
    first = A.orthogonalize(x)
    out = torch.empty_like(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert A.orthogonalize(x, out=out, stream=side) is out
    with torch.cuda.stream(side):
        other = A.orthogonalize(x)
    torch.cuda.synchronize()
    assert torch.equal(first, out) and torch.equal(first, other)


@pytest.mark.parametrize("shape", [(300, 6000), (140, 4100), (1500, 2100), (1030, 1030)],
                         ids=lambda s: "x".join(map(str, s)))
def test_parts_of_tiles_give_the_same_bits(shape):
    """Whichever part comes last: alone, and beside a call that takes SMs away."""
    x = momentum_like(*shape, _gen(9))
    first = A.orthogonalize(x)
    _check(x, first)
    other = torch.stack([momentum_like(300, 400, _gen(i)) for i in range(20)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(6):
        A.orthogonalize(other, stream=side)
        outs.append(A.orthogonalize(x))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


def test_captured_calls_have_scratch_of_their_own():
    xs = [momentum_like(300, 200, _gen(i)) for i in range(2)]
    want = [A.orthogonalize(x) for x in xs]
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(A.orthogonalize(x))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_rows_behind_the_last_are_left_alone():
    x = momentum_like(130, 67, _gen(6))
    field = torch.full((130 * 67 + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = field[32:-32].view(130, 67)
    A.orthogonalize(x, out=out)
    assert (field[:32] == 7).all() and (field[-32:] == 7).all()
    _check(x, out)


def test_empty():
    for shape in ((0, 5), (5, 0), (0, 4, 4), (3, 0, 4)):
        assert A.orthogonalize(torch.empty(shape, device="cuda")).shape == shape


@pytest.mark.parametrize("shape", [(3, 140, 500), (3, 40, 200), (2, 40, 900)],
                         ids=lambda s: "x".join(map(str, s)))
def test_a_copy_or_product_that_never_comes_ends_in_nan(shape):
    x = torch.stack([momentum_like(*shape[1:], _gen(i)) for i in range(shape[0])])
    want = A.orthogonalize(x)
    A.test_stall_tile(1)
    out = A.orthogonalize(x)
    torch.cuda.synchronize()
    assert out.isnan().any()
    assert torch.equal(A.orthogonalize(x), want)


def test_factor_is_nearly_orthogonal():
    """Singular values come near 1 (0.68 to 1.13 after these steps)."""
    x = momentum_like(96, 400, _gen(7))
    s = torch.linalg.svdvals(A.orthogonalize(x).double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25
    assert torch.allclose(s, torch.linalg.svdvals(exact(x)), atol=0.02)
