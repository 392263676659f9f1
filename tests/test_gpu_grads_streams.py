"""One list of gradients on several streams at once: calls that overlap on the
GPU keep apart, as Python calls (which bring scratch of their own) and through
the C entry points that take scratch."""
import ctypes
import gc

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _tensors(sizes, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * 1e-2).to(
        (torch.float32, torch.bfloat16)[i % 2]) for i, n in enumerate(sizes)]


@pytest.mark.parametrize("sizes", [[5000, 77], [3_000_001, 17, 400_000], [50_000_000, 12_345_678]],
                         ids=["small", "middle", "large"])
def test_norms_and_clips_on_alternating_streams(sizes):
    """Norms and clips by different thresholds, none waiting for another."""
    g = A.GradList(_tensors(sizes, 1))
    flat = torch.cat([t.reshape(-1).float() for t in g.tensors])
    norm = A.grad_norm(g)
    n = float(norm)
    assert abs(n - float(flat.double().norm())) <= 17 * U * n
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty(g.numel, device="cuda") for _ in streams]
    limits = [n / 2, n / 8, 2 * n]
    want = []
    for m in limits:
        o = torch.empty(g.numel, device="cuda")
        A.clip_grads(g, m, out=o)
        want.append(o)
    torch.cuda.synchronize()
    norms = []
    for _ in range(60):
        for s, o, m in zip(streams, outs, limits):
            norms.append(A.clip_grads(g, m, out=o, stream=s))
            norms.append(A.grad_norm(g, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(norm, v) for v in norms)
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    # and no call that follows suffers
    assert all(torch.equal(norm, A.grad_norm(g)) for _ in range(3))


def test_a_captured_call_beside_others():
    """A graph replayed on one stream while others use the same list."""
    g = A.GradList(_tensors([2_000_003, 1001], 2))
    out = torch.empty(g.numel, device="cuda")
    norm = A.grad_norm(g)
    limit = float(norm) / 2
    A.clip_grads(g, limit, out=out)
    want = out.clone()
    graph, one, other = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        inside = A.clip_grads(g, limit, out=out)
    torch.cuda.synchronize()
    norms = []
    for _ in range(40):
        with torch.cuda.stream(one):
            graph.replay()
        norms += [A.grad_norm(g, stream=other), A.grad_norm(g)]
    torch.cuda.synchronize()
    assert all(torch.equal(norm, v) for v in norms + [inside])
    assert torch.equal(out, want)


def test_the_entry_points_with_scratch():
    """Zeroed scratch of exactly the size asked for, call after call; the handle's
    own without; and what is refused."""
    ts = _tensors([40_000, 9], 3)
    g = A.GradList(ts)
    lib, need = A.load(), A.load().aloco_grads_scratch_bytes(g._handle)
    norm, want = torch.zeros((), device="cuda"), A.grad_norm(g)
    opts = ctypes.byref(A.Opts(stream=torch.cuda.current_stream().cuda_stream))
    assert lib.aloco_grads_scratch_bytes(None) == 0
    buf = torch.full((need + 64,), 90, dtype=torch.uint8, device="cuda")
    buf[32:32 + need] = 0
    for _ in range(3):
        norm.zero_()
        assert lib.aloco_grad_norm_in(g._handle, norm.data_ptr(), buf[32:].data_ptr(), need,
                                      opts) == A.OK
        torch.cuda.synchronize()
        assert torch.equal(norm, want)
        assert bool((buf[:32] == 90).all()) and bool((buf[32 + need:] == 90).all())
    for call in (lambda: lib.aloco_grad_norm(g._handle, norm.data_ptr(), opts),
                 lambda: lib.aloco_clip_grads(g._handle, 1e3, None, 0, norm.data_ptr(), opts)):
        norm.zero_()
        assert call() == A.OK
        torch.cuda.synchronize()
        assert torch.equal(norm, want)
    out = torch.zeros(g.numel, device="cuda")
    at = buf[32:].data_ptr()
    clip = lambda o, s, b: lib.aloco_clip_grads_in(g._handle, 1.0, o, 0, norm.data_ptr(), s, b, opts)
    assert clip(out.data_ptr(), at, need - 1) == A.ERR_ARG and "scratch" in A.last_error()
    assert clip(out.data_ptr(), at + 8, need) == A.ERR_ARG and "scratch" in A.last_error()
    assert clip(out.data_ptr(), ts[0].data_ptr(), need) == A.ERR_ALIAS
    assert clip(out.data_ptr(), out.data_ptr(), need) == A.ERR_ALIAS
    host = torch.zeros(need + 16, dtype=torch.uint8)
    assert clip(out.data_ptr(), (host.data_ptr() + 15) // 16 * 16, need) != A.OK
    assert clip(out.data_ptr(), at, need) == A.OK


def test_lists_dropped_while_a_graph_is_captured():
    """Also one that only the collector finds: the capture goes on, the graph is
    right, and the memory goes back when another list is made."""
    g = A.GradList(_tensors([4000, 9], 4))
    want = A.grad_norm(g)
    for cycle in (False, True):
        other = A.GradList(_tensors([500], 5))
        A.grad_norm(other)
        if cycle:
            other.itself = other
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        gc.collect()
        with torch.cuda.graph(graph):
            norm = A.grad_norm(g)
            del other
            gc.collect()
            again = A.grad_norm(g)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and torch.equal(again, want)
    assert A._dropped_lists
    assert torch.equal(A.grad_norm(A.GradList(g.tensors)), want)
    del g
    gc.collect()
