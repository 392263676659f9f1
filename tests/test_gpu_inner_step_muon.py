"""An inner step of post-training with the token scores and the orthogonalised
update, as a training loop runs them: the example, and the chain of calls against
the same in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A
from _orthogonal import allowed

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "post_training", os.path.join(ROOT, "examples", "post_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kw", [dict(optimizer="muon"), dict(optimizer="muon", entropy=0.01),
                                dict(entropy=0.01), dict(loss="preference", optimizer="muon")],
                         ids=lambda k: "-".join(map(str, k.values())))
def test_example_runs(kw):
    got = _example().run(rounds=2, steps=3, **kw)
    assert len(got) == 2 and all(math.isfinite(m) for m in got)


def test_entropy_gradient_of_the_example_equals_autograd():
    ex = _example()
    gen = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn(64, 96, generator=gen, device="cuda")
    tok = torch.randint(0, 96, (64,), generator=gen, device="cuda")
    g, h = ex.entropy_grad(logits, tok, 0.1)
    y = logits.double().requires_grad_()
    entropy = torch.special.entr(torch.softmax(y, -1)).sum(-1).mean()
    (-0.1 * entropy).backward()
    entropy = entropy.detach()
    # log p and H in fp32: 1e-5 and 2e-5 (1 + H) of p / rows
    assert abs(float(h) - float(entropy)) <= 2e-5 * (1 + float(entropy))
    tol = 0.1 / 64 * torch.softmax(y.detach(), -1) * 4e-5 * (1 + float(entropy)) + 2.0 ** -22 * \
        y.grad.abs()
    assert ((g.double() - y.grad).abs() <= tol).all()


def _layout(vocab, dim):
    """E and W as matrices, with a vector of biases between them."""
    return [(0, vocab, dim), (vocab * dim + vocab, dim, vocab)], vocab * dim, 2 * vocab * dim + vocab


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "graph"])
def test_the_chain_of_calls(captured):
    """Scores of three workers' tokens, the gradient of a loss over all of them,
    clipping into flat vectors, one muon_step for the matrices of all workers and
    one adamw_step for the biases between them."""
    vocab, dim, rows, M = 300, 140, 96, 3
    parts, cut, n = _layout(vocab, dim)
    gen = torch.Generator("cuda").manual_seed(7)
    xs = [0.1 * torch.randn(n, generator=gen, device="cuda") for _ in range(M)]
    bufs = [1e-2 * torch.randn(n, generator=gen, device="cuda") for _ in range(M)]
    m1, m2 = ([torch.zeros(vocab, device="cuda") for _ in range(M)] for _ in range(2))
    ctx = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    tok = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    by_logp = torch.randn(rows, generator=gen, device="cuda") / rows
    by_h = torch.randn(rows, generator=gen, device="cuda") / rows
    by_top = torch.randn(rows, 4, generator=gen, device="cuda") / rows
    flats = [torch.empty(n, device="cuda") for _ in range(M)]
    muon = A.muon_cfg(lr=1e-2)
    matrices = A.Matrices(parts)
    adam = A.adamw_cfg(lr=1e-2, weight_decay=0.0, max_grad_norm=0.0, step=1)
    lists = [A.GradList([torch.zeros(s, device="cuda") for s in
                         ((vocab, dim), (vocab,), (dim, vocab))]) for _ in range(M)]
    before = [(x.clone(), b.clone()) for x, b in zip(xs, bufs)]

    def views(x):
        return x[:cut].view(vocab, dim), x[cut:cut + vocab], x[cut + vocab:].view(dim, vocab)

    def step():
        for x, grads, flat in zip(xs, lists, flats):
            E, bias, W = views(x)
            logits = E[ctx] @ W + bias
            s = A.token_scores(logits, tok, top=4)
            g = A.token_scores_grad(logits, tok, s, d_logp=by_logp, d_entropy=by_h, d_top=by_top)
            grads.tensors[0].zero_().index_add_(0, ctx, g @ W.T)
            grads.tensors[1].copy_(g.sum(0))
            grads.tensors[2].copy_(E[ctx].T @ g)
            A.clip_grads(grads, 1.0, out=flat)
        A.muon_step(xs, flats, bufs, matrices, muon)
        A.adamw_step([x[cut:cut + vocab] for x in xs], [f[cut:cut + vocab] for f in flats], m1, m2,
                     adam, want_stats=False)

    if captured:
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()                     # (what is made on first use)
        torch.cuda.synchronize()
        for x, b, (x0, b0) in zip(xs, bufs, before):
            x.copy_(x0)
            b.copy_(b0)
        for t in (*m1, *m2):
            t.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for x, b, (x0, b0) in zip(xs, bufs, before):
            x.copy_(x0)
            b.copy_(b0)
        for t in (*m1, *m2):
            t.zero_()
        graph.replay()
    else:
        step()
    torch.cuda.synchronize()

    for x, b, (x0, b0) in zip(xs, bufs, before):
        E, bias, W = (v.double().requires_grad_() for v in views(x0))
        lp = torch.log_softmax(E[ctx] @ W + bias, -1)
        ids = lp.topk(4, -1)[1]
        loss = (lp.gather(1, tok[:, None])[:, 0] * by_logp).sum() + \
            (torch.special.entr(lp.exp()).sum(-1) * by_h).sum() + (lp.gather(1, ids) * by_top).sum()
        loss.backward()
        flat = torch.cat([E.grad.reshape(-1), bias.grad, W.grad.reshape(-1)])
        flat = flat * min(1.0, 1.0 / (float(flat.norm()) + 1e-6))
        for at, r, c in parts:
            part = slice(at, at + r * c)
            want_b = 0.95 * b0[part].double() + flat[part]
            # products over at most 300 terms in fp32, and the scores' 1e-5
            assert float((b[part] - want_b).norm()) <= 1e-4 * float(want_b.norm())
            o, off = allowed((flat[part] + 0.95 * want_b).view(r, c))
            step_size = 1e-2 * 0.2 * math.sqrt(max(r, c))
            theta = (1 - 1e-3) * x0[part].double() - step_size * o.reshape(-1)
            # 1e-4 in the gradient grows at most with the steps' slope, 3.4445^5 = 485
            tol = step_size * (off + 485 * 1e-4) + 2.0 ** -22 * float(theta.norm())
            assert float((x[part] - theta).norm()) <= tol
        part = slice(cut, cut + vocab)
        assert torch.equal(b[part], b0[part])
        want = x0[part].double() - 1e-2 * flat[part] / (flat[part].abs() + 1e-8)
        assert ((x[part] - want).abs() <= 1e-2 * 1e-2).all()
