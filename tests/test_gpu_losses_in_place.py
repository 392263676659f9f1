"""The post-training losses over many rows: gradients written over the logits
while later rows are fetched ahead, calls of more than 80 MB in graphs and on two
streams, and values without a gradient.

All of them against the same kernels on buffers of their own, which tests/
test_gpu_losses.py holds against float64: bit for bit."""
import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

BOTH = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]
# odd vocabularies, whose rows share 16-byte units with their neighbours: several
# rows for every block and cluster, below and above 80 MB, one CTA a row to eight
SHAPES = [(4000, 501), (6000, 2301), (4000, 5003), (3000, 16001), (2000, 40011), (700, 128257)]


def _inputs(n, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.empty(n, V, dtype=dtype, device="cuda").normal_(0, 2, generator=g)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    t[5::11] = -1
    lp = A.token_logprobs(x, t)
    f = lambda s: torch.randn(n, generator=g, device="cuda") * s
    w = torch.full((n,), 1.0 / n, device="cuda")
    w[3::7] = 0.0
    return dict(x=x, t=t, adv=f(1.0), old=lp + f(0.2), ref=lp + f(0.2), w=w,
                cu=torch.linspace(0, n, 2 * 24 + 1, device="cuda").long())


def _policy(i, **kw):
    return A.policy_loss(i["x"], i["t"], i["adv"], i["old"], i["w"], ref_logp=i["ref"],
                         kl_coef=0.05, **kw)


def _pref(i, **kw):
    return A.preference_loss(i["x"], i["t"], i["cu"], i["ref"], label_smoothing=0.1, **kw)


def _same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,V", SHAPES)
def test_the_gradient_over_the_logits_of_many_rows(n, V, dtype):
    i = _inputs(n, V, dtype, V)
    x0 = i["x"].clone()
    for call in (_policy, _pref):
        want = call(i)
        assert torch.equal(i["x"], x0) and bool(torch.isfinite(want.grad).all())
        for _ in range(3):
            got = call(i, grad=i["x"])
            assert got.grad.data_ptr() == i["x"].data_ptr() and _same(got, want)
            i["x"].copy_(x0)


@pytest.mark.parametrize("how", ["shifted", "by_position"])
@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_the_gradient_over_a_view_of_the_logits(dtype, how):
    """A view without each sequence's last position, and one that lies position by
    position; what the view leaves out keeps its values."""
    B, T, V = 6, 400, 8003
    i = _inputs(B * T, V, dtype, 9)
    rest = torch.full((B, T + 1, V), 3.0, dtype=dtype, device="cuda")
    if how == "shifted":
        lay = lambda full: full[:, :T]
    else:
        lay = lambda full: full.view(T + 1, B, V)[:T].transpose(0, 1)
    own, full = rest.clone(), rest.clone()
    x = lay(full)
    j = {k: v if k in ("x", "cu") else v.view(B, T) for k, v in i.items()}
    j["x"] = x
    for call in (_policy, _pref):
        x.copy_(i["x"].view(B, T, V))
        want = call(j, grad=lay(own))
        got = call(j, grad=x)
        assert _same(got, want) and torch.equal(full, own)
        kept = full[:, T] if how == "shifted" else full.view(T + 1, B, V)[T]
        assert bool((kept == 3.0).all())


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
def test_large_calls_in_a_graph(dtype):
    """Over 80 MB the policy loss's sums, and beyond 2048 rows the pairs, are
    kernels of their own: captured, and replayed on other logits."""
    i = _inputs(2600, 16500, dtype, 3)
    _policy(i), _pref(i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [*_policy(i), *_pref(i)]
    for seed in (4, 5):
        i["x"].copy_(_inputs(2600, 16500, dtype, seed)["x"])
        graph.replay()
        torch.cuda.synchronize()
        assert _same(got, [*_policy(i), *_pref(i)])


def test_large_calls_on_two_streams_at_once():
    jobs = []
    for k in range(2):
        i = _inputs(2500, 17003, torch.bfloat16, 30 + k)
        jobs.append((i, [*_policy(i), *_pref(i)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        for i, want, s in jobs:
            got.append(([*_policy(i, stream=s), *_pref(i, stream=s)], want))
    torch.cuda.synchronize()
    assert all(_same(a, b) for a, b in got)


@pytest.mark.parametrize("dtype", BOTH, ids=IDS)
@pytest.mark.parametrize("n,V", SHAPES)
def test_values_without_a_gradient(n, V, dtype):
    i = _inputs(n, V, dtype, V + 1)
    for call in (_policy, _pref):
        want, got = call(i), call(i, want_grad=False)
        assert got.grad is None and _same(got[:-1], want[:-1])
