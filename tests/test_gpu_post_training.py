"""The post-training operators together, as a training loop uses them: the
example's inner steps and outer rounds improve what they train for."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "post_training", os.path.join(ROOT, "examples", "post_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("loss,gain", [("policy", 0.3), ("preference", 0.1)])
def test_rounds_improve_what_they_train_for(loss, gain):
    got = _example().run(loss)
    assert got[-1] > got[0] + gain, got


def test_a_step_equals_autograd():
    """E's and W's gradients of one policy step, against torch's autograd of the
    same loss in fp32 (the logits are rounded to bf16 on the way: 2^-8 of the
    gradient's scale)."""
    ex = _example()
    from paper_2609_36662_gb300 import aloco as A
    gen = torch.Generator("cuda").manual_seed(3)
    theta = torch.randn(2 * 96 * 16, generator=gen, device="cuda") / 4
    w = ex.Worker(theta, 96, 16, 1)
    ctx = torch.randint(0, 96, (64,), generator=gen, device="cuda")
    tok = torch.randint(0, 96, (64,), generator=gen, device="cuda")
    adv = torch.randn(64, generator=gen, device="cuda")
    logits = w.logits(ctx)
    old = A.token_logprobs(logits, tok)
    r = A.policy_loss(logits, tok, adv, old, torch.full_like(adv, 1 / 64), ref_logp=old,
                      kl_coef=0.1)
    w.backward(ctx, r.grad)
    E, W = w.E.clone().requires_grad_(), w.W.clone().requires_grad_()
    lp = torch.log_softmax(E[ctx] @ W.T, -1).gather(1, tok[:, None])[:, 0]
    ratio = torch.exp(lp - lp.detach())
    (-(ratio * adv).sum() / 64).backward()
    for got, want in ((w.gE, E.grad), (w.gW.float(), W.grad)):
        assert float((got - want).norm() / want.norm()) < 2.0 ** -6
