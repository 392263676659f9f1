"""Post-training with outer synchronisation: M workers tune a small policy, each
on its own data, with AutoLoCo rounds between intervals of inner steps.

    python examples/post_training.py [--loss policy|preference] [--rounds 6]
                                     [--optimizer adamw|muon] [--entropy 0.01]

The policy is a next-token model that one matrix product makes of an embedding:
logits = E[context] W^T.  An answer is a token; the reward of (context, token)
is a fixed random score.  Every inner step of a worker is

    logits           torch
    loss, gradient   aloco.policy_loss or aloco.preference_loss, with the old
                     and the reference policy scored by aloco.token_logprobs
    entropy bonus    aloco.token_scores and aloco.token_scores_grad (policy, with
                     --entropy)
    E, W gradients   torch
    clipping         aloco.clip_grads, into the flat vector of the replica
    update           aloco.adamw_step, or aloco.muon_step for both matrices

and every interval ends with aloco.sync over the workers' replicas.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_36662_gb300 import aloco as A  # noqa: E402


class Worker:
    """A replica: one flat fp32 vector that holds E and W, its AdamW state, and
    the gradient list of its two matrices."""

    def __init__(self, theta, vocab, dim, seed, optimizer="adamw"):
        self.optimizer = optimizer
        self.matrices = A.Matrices([(0, vocab, dim), (vocab * dim, vocab, dim)])
        self.x = theta.clone()
        self.E, self.W = self.x.view(2, vocab, dim)
        self.m, self.v = torch.zeros_like(theta), torch.zeros_like(theta)
        self.gE = torch.empty(vocab, dim, device="cuda")
        self.gW = torch.empty(vocab, dim, device="cuda", dtype=torch.bfloat16)
        self.grads = A.GradList([self.gE, self.gW])
        self.flat = torch.empty_like(theta)
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.steps = 0

    def logits(self, ctx):
        return (self.E[ctx] @ self.W.T).to(torch.bfloat16)

    def backward(self, ctx, by_logits):
        """Gradients of E and W from the gradient by the logits."""
        g = by_logits.float()
        self.gW.copy_(g.T @ self.E[ctx])
        self.gE.zero_().index_add_(0, ctx, g @ self.W)

    def update(self, lr):
        self.steps += 1
        norm = A.clip_grads(self.grads, 1.0, out=self.flat)
        if self.optimizer == "muon":
            # (the factor has no scale of its own: steps as long as AdamW's)
            A.muon_step([self.x], [self.flat], [self.m], self.matrices,
                        A.muon_cfg(lr=lr, momentum=0.9, weight_decay=0.0))
            return norm
        cfg = A.adamw_cfg(lr=lr, beta2=0.999, weight_decay=0.0, max_grad_norm=0.0,
                          step=self.steps)
        A.adamw_step([self.x], [self.flat], [self.m], [self.v], cfg, want_stats=False)
        return norm


def entropy_grad(logits, token, coef):
    """The gradient by the logits of -coef times the mean entropy, and that mean."""
    s = A.token_scores(logits, token)
    each = torch.full_like(s.entropy, -coef / token.numel())
    return A.token_scores_grad(logits, token, s, d_entropy=each), s.entropy.mean()


def policy_step(w, ref, score, batch, lr, entropy=0.0):
    """One sampled answer per context; the advantage is its reward against the
    batch's mean."""
    vocab = score.shape[1]
    ctx = torch.randint(0, vocab, (batch,), generator=w.gen, device="cuda")
    old = w.logits(ctx)
    token = torch.multinomial(torch.softmax(old.float(), -1), 1, generator=w.gen)[:, 0]
    reward = score[ctx, token]
    adv = (reward - reward.mean()) / (reward.std() + 1e-6)
    old_logp = A.token_logprobs(old, token)
    ref_logp = A.token_logprobs(ref.logits(ctx), token)
    weight = torch.full_like(adv, 1.0 / batch)
    for _ in range(2):  # the second step's ratios have left 1
        logits = w.logits(ctx)
        bonus = entropy_grad(logits, token, entropy)[0] if entropy else None
        r = A.policy_loss(logits, token, adv, old_logp, weight, ref_logp=ref_logp, kl_coef=0.01,
                          grad=logits)
        w.backward(ctx, r.grad if bonus is None else r.grad + bonus)
        w.update(lr)
    return reward.mean(), r.terms[0]


def preference_step(w, ref, score, batch, lr, entropy=0.0):
    """Pairs of two-token answers, the better one by its reward first."""
    vocab = score.shape[1]
    ctx = torch.randint(0, vocab, (batch, 2), generator=w.gen, device="cuda")
    tokens = torch.randint(0, vocab, (batch, 2, 2), generator=w.gen, device="cuda")
    reward = score[ctx[:, None, :], tokens].sum(-1)
    first = reward.argmax(1)
    order = torch.stack([first, 1 - first], 1)
    tokens = torch.gather(tokens, 1, order[:, :, None].expand(-1, -1, 2)).reshape(-1)
    ctx = ctx[:, None, :].expand(-1, 2, -1).reshape(-1)
    cu = torch.arange(0, 4 * batch + 1, 2, device="cuda", dtype=torch.int32)
    logits = w.logits(ctx)
    r = A.preference_loss(logits, tokens, cu, A.token_logprobs(ref.logits(ctx), tokens), beta=0.5,
                          grad=logits)
    w.backward(ctx, r.grad)
    w.update(lr)
    return (r.log_ratios[0::2] > r.log_ratios[1::2]).float().mean(), r.loss


def run(loss="policy", workers=4, vocab=512, dim=64, batch=1024, rounds=6, steps=25, lr=5e-3,
        seed=0, optimizer="adamw", entropy=0.0):
    """The rounds' measures: the mean reward of sampled answers (policy), or the
    share of pairs that the policy orders as the reference's judge does."""
    gen = torch.Generator("cuda").manual_seed(seed)
    theta = torch.randn(2 * vocab * dim, generator=gen, device="cuda") / math.sqrt(dim)
    momentum = torch.zeros_like(theta)
    score = torch.randn(vocab, 32, generator=gen, device="cuda") @ \
        torch.randn(32, vocab, generator=gen, device="cuda") / math.sqrt(32)
    ref = Worker(theta, vocab, dim, 0)
    team = [Worker(theta, vocab, dim, 1 + i, optimizer) for i in range(workers)]
    schedule = A.Schedule.make(A.SCHED_CONSTANT, lr, lr, 0, 1)
    step = policy_step if loss == "policy" else preference_step
    measures = []
    for k in range(rounds):
        got = [[step(w, ref, score, batch, lr, entropy) for _ in range(steps)] for w in team]
        st = A.sync(theta, momentum, [w.x for w in team], H_sel=steps, H_base=steps,
                    step=k * steps, schedule=schedule, outer_lr=0.7, outer_beta=0.6)
        measures.append(float(sum(m for g in got for m, _ in g)) / (steps * workers))
        print(f"round {k + 1}: {'reward' if loss == 'policy' else 'ordered'} {measures[-1]:.3f}  "
              f"loss {float(got[0][-1][1]):.4f}  D {st['D']:.3e}  C {st['C']:.3f}")
    return measures


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--loss", choices=["policy", "preference"], default="policy")
    p.add_argument("--rounds", type=int, default=6)
    p.add_argument("--optimizer", choices=["adamw", "muon"], default="adamw")
    p.add_argument("--entropy", type=float, default=0.0)
    a = p.parse_args()
    run(a.loss, rounds=a.rounds, optimizer=a.optimizer, entropy=a.entropy)
