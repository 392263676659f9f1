"""The post-training operators, as cases that can be timed and checked.

A worker's inner step in preference or policy tuning goes from logits to a
loss and its gradient, and from the parameters' gradients to a clipped vector
that the optimizer takes.  The calls are

  logp     aloco.token_logprobs    log-probabilities of given tokens
  policy   aloco.policy_loss       clipped policy loss with a KL term, with
                                   the gradient by the logits
  pref     aloco.preference_loss   loss of paired log ratios, with the
                                   gradient by the logits
  norm     aloco.grad_norm         global norm of many gradient tensors
  clip     aloco.clip_grads        the same, clipped into one flat vector

With `own` false the same results come from elementary torch operations in 32
bits; with `own` true from the package's kernels.
"""
import math

import torch

own = False

# Largest work of any case, listed or drawn (bytes read and written).
MOST_BYTES = 4.4e9

BETA, SMOOTH = 0.1, 0.05
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
MAX_NORM = 1.0


def listed():
    return [
        # One sampled token is scored as it comes: launches and host work.
        {"name": "logp_one", "kind": "logp", "b": 1, "l": 1, "v": 32000, "x": "bf16",
         "temp": 1.0, "shift": 0, "prompt": 0.0, "banned": False},
        # A reference model's pass over four sequences at the fine-tuning
        # model's vocabulary: the logits of positions 0..l-1 score the tokens
        # 1..l, a view that leaves out each sequence's last row.
        {"name": "logp_128k", "kind": "logp", "b": 4, "l": 1023, "v": 128256, "x": "bf16",
         "temp": 1.0, "shift": 1, "prompt": 0.25, "banned": False},
        # A micro-batch of a few dozen tokens with logits kept in fp32.
        {"name": "policy_tiny", "kind": "policy", "b": 3, "l": 16, "v": 32000, "x": "f32",
         "temp": 1.0, "shift": 0, "prompt": 0.25, "banned": False},
        # An ordinary worker's batch: eight sequences of 1024 positions, half
        # of them prompt.
        {"name": "policy_32k", "kind": "policy", "b": 8, "l": 1023, "v": 32000, "x": "bf16",
         "temp": 1.0, "shift": 1, "prompt": 0.5, "banned": False},
        # An odd vocabulary in fp32 (no row after the first starts on a
        # 16-byte boundary), sampled at a temperature and with banned tokens.
        {"name": "policy_odd", "kind": "policy", "b": 3, "l": 511, "v": 50257, "x": "f32",
         "temp": 0.7, "shift": 0, "prompt": 0.1, "banned": True},
        # Eight sequences at the fine-tuning model's vocabulary: the largest.
        {"name": "policy_128k", "kind": "policy", "b": 8, "l": 1000, "v": 128256, "x": "bf16",
         "temp": 1.0, "shift": 0, "prompt": 0.1, "banned": False},
        # Two short pairs.
        {"name": "pref_small", "kind": "pref", "pairs": 2, "l": 95, "v": 32000, "x": "bf16",
         "temp": 1.0, "prompt": 0.25, "banned": False},
        # A worker's batch of eight pairs with ragged lengths up to 1024.
        {"name": "pref_32k", "kind": "pref", "pairs": 8, "l": 1024, "v": 32000, "x": "bf16",
         "temp": 1.0, "prompt": 0.25, "banned": False},
        # The gradients of the 150M set, tensor by tensor, in fp32.
        {"name": "norm_150m", "kind": "norm", "set": "llama150m", "n": 0, "x": "f32"},
        # A small model's gradients in mixed types, as views that start at odd
        # elements, with vectors, single values and empty tensors among them.
        {"name": "norm_odd", "kind": "norm", "set": "odd", "n": 3_000_017, "x": "mixed"},
        # The gradients of the 1.1B set, clipped into the optimizer's vector.
        {"name": "clip_1b", "kind": "clip", "set": "llama1b", "n": 0, "x": "bf16",
         "out": "bf16"},
        # The small model's again, clipped into an fp32 vector.
        {"name": "clip_odd", "kind": "clip", "set": "odd", "n": 7_000_003, "x": "mixed",
         "out": "f32"},
    ]


def draw(rng):
    kind = rng.choice(["logp", "policy", "policy", "pref", "pref", "norm", "clip"])
    x = rng.choice(["f32", "bf16"])
    if kind in ("norm", "clip"):
        c = {"kind": kind, "set": "odd", "n": _size(rng, 50_000, 1e9),
             "x": rng.choice(["f32", "bf16", "mixed"])}
        if kind == "clip":
            c["out"] = rng.choice(["f32", "bf16"])
        while work(c)["bytes"] > MOST_BYTES:
            c["n"] = c["n"] * 2 // 3
        return c
    v = rng.choice([32000, 128256, _size(rng, 500, 131072), _size(rng, 500, 131072)])
    c = {"kind": kind, "v": v, "x": x, "temp": rng.choice([1.0, 1.0, 0.7, 1.3]),
         "prompt": rng.choice([0.0, 0.1, 0.25, 0.5]), "banned": rng.random() < 0.5}
    c["l"] = _size(rng, 2, 2048)
    if kind == "pref":
        c["pairs"] = _size(rng, 1, 16)
    else:
        c["b"] = _size(rng, 1, 16)
        c["shift"] = rng.choice([0, 1])
    while work(c)["bytes"] > MOST_BYTES:
        c["l"] = c["l"] * 2 // 3
    return c


def _size(rng, lo, hi):
    """Log-uniform; one in three larger sizes is a multiple of 64."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    return n // 64 * 64 if n > 640 and rng.random() < 1 / 3 else n


# ------------------------------------------------------------------- shapes

def _prompt(length, case):
    """Leading positions of a sequence that carry no loss."""
    return int(length * case["prompt"])


def _lens(case):
    """Lengths of the chosen and rejected sequences in turn: ragged between
    half of l and l."""
    lo = (case["l"] + 1) // 2
    return [lo + (i * 7919 + 13) % (case["l"] - lo + 1) for i in range(2 * case["pairs"])]


def _llama(layers, d, kv, ffn, vocab, tied):
    """Tensor sizes of a Llama-style set, in packing order."""
    layer = [d, d * d, d * kv, d * kv, d * d, d, d * ffn, d * ffn, ffn * d]
    return [vocab * d] + layer * layers + [d] + ([] if tied else [vocab * d])


def _sizes(case):
    if case["set"] == "llama150m":
        return _llama(12, 768, 768, 3072, 32000, True)
    if case["set"] == "llama1b":
        return _llama(22, 2048, 256, 5632, 32000, False)
    unit = max(1, case["n"] // 1_600_000)
    cycle = [150_000 * unit, 769, 50_257 * unit, 1, 0, 12_289 * unit, 4096]
    out, left = [], case["n"]
    while left:
        out.append(min(left, cycle[len(out) % len(cycle)]))
        left -= out[-1]
    return out


def _elt(case, i=0):
    """Bytes of an element of tensor i."""
    return {"f32": 4, "bf16": 2, "mixed": 4 if i % 5 == 1 else 2}[case["x"]]


def work(case):
    if case["kind"] in ("norm", "clip"):
        sizes = _sizes(case)
        read = sum(n * _elt(case, i) for i, n in enumerate(sizes))
        n = sum(sizes)
        if case["kind"] == "norm":
            return {"bytes": read + 4, "flops": 2 * n}
        return {"bytes": read + n * (4 if case["out"] == "f32" else 2) + 4, "flops": 3 * n}
    if case["kind"] == "pref":
        lens = _lens(case)
        rows = sum(lens)
        live = rows - sum(_prompt(n, case) for n in lens)
    else:
        rows = case["b"] * case["l"]
        live = rows - case["b"] * _prompt(case["l"], case)
    row = case["v"] * _elt(case)
    if case["kind"] == "logp":
        return {"bytes": live * row + rows * 12, "flops": 4 * live * case["v"]}
    # logits of the rows that count in, a whole gradient out; the rest is the
    # tokens and a few floats a row
    return {"bytes": live * row + rows * row + rows * 28, "flops": 7 * live * case["v"]}


# ------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _uniform(shape, lo, hi, gen):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=gen)


def _normal(shape, std, gen):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)


def _logits(case, full, v, gen):
    """Logits spread as a trained model's, in place, with the tokens that were
    drawn from them well above the rest (-0.1 to -6 in log-probability)."""
    full.normal_(0.0, 2.0, generator=gen)
    if case["banned"]:
        full[..., v // 3:v // 3 + 17] = -math.inf
        full[..., v - v // 50:] = torch.finfo(full.dtype).min
    t = torch.randint(0, v, full.shape[:-1], generator=gen, device="cuda")
    top = math.log(v) + 1.5
    full.scatter_(-1, t.unsqueeze(-1),
                  _uniform(t.shape + (1,), top - 2.5, top + 4.0, gen).to(full.dtype))
    return t


def _tokens_logp(x, t, case):
    lse = torch.cat([torch.logsumexp(r.float() / case["temp"], -1)
                     for r in x.split(1 if x.dim() == 3 else 1024)])
    return x.gather(-1, t.unsqueeze(-1)).squeeze(-1).float() / case["temp"] - lse


def _old(lp, gen):
    """The sampling policy's log-probabilities; no ratio is left so near an
    edge of the clipping range that rounding decides on which side it lies."""
    old = lp + _normal(lp.shape, 0.15, gen)
    for edge in (1 - CLIP_LOW, 1 + CLIP_HIGH):
        old += 0.01 * (torch.abs(torch.exp(lp - old) - edge) < 2e-3)
    return old


def prepare(case, seed):
    gen = _gen(seed)
    if case["kind"] in ("norm", "clip"):
        return _prepare_grads(case, gen)
    dtype = torch.float32 if case["x"] == "f32" else torch.bfloat16
    v = case["v"]
    if case["kind"] == "pref":
        lens = _lens(case)
        x = torch.empty(sum(lens), v, dtype=dtype, device="cuda")
        t = _logits(case, x, v, gen)
        starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
        seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
        # one answer of a pair has gained on the reference, the other lost
        ref = _tokens_logp(x, t, case) + _normal(t.shape, 0.25, gen) + \
            _normal(len(lens), 0.02, gen)[seq]
        live = torch.cat([torch.arange(n) >= _prompt(n, case) for n in lens]).cuda()
        return {"kind": "pref", "case": case, "x": x, "t": torch.where(live, t, -1), "ref": ref,
                "cu": torch.tensor(starts, dtype=torch.int32, device="cuda"), "seq": seq}
    b, l = case["b"], case["l"]
    full = torch.empty(b, l + case["shift"], v, dtype=dtype, device="cuda")
    t = _logits(case, full, v, gen)[:, :l].contiguous()
    x = full[:, :l]
    q = _prompt(l, case)
    if case["kind"] == "logp":
        t[:, :q] = -1
        return {"kind": "logp", "case": case, "x": x, "t": t}
    lp = _tokens_logp(x, t, case)
    s = {"kind": "policy", "case": case, "x": x, "t": t, "old": _old(lp, gen),
         "ref": lp + _normal(lp.shape, 0.3, gen),
         "adv": _normal((b, 1), 1.0, gen) + _normal((b, l), 0.1, gen)}
    w = torch.ones(b, l, device="cuda")
    w[:, :q] = 0.0
    s["w"] = w / w.sum()
    if case["banned"]:
        # what a prompt's rows hold is nobody's business
        x[:, :q] = math.nan
    return s


def _prepare_grads(case, gen):
    """Gradients whose norm is some times the clipping threshold; the tensors
    of an odd set are views into one buffer of their type, one behind the
    other."""
    sizes = _sizes(case)
    n = sum(sizes)
    std = 3.0 * MAX_NORM / math.sqrt(n)
    kinds = [torch.float32 if _elt(case, i) == 4 else torch.bfloat16 for i in range(len(sizes))]
    if case["set"] == "odd":
        at, ts = {torch.float32: 1, torch.bfloat16: 1}, []
        base = {k: torch.empty(1 + sum(m for m, q in zip(sizes, kinds) if q == k), dtype=k,
                               device="cuda").normal_(0.0, std, generator=gen) for k in at}
        for m, k in zip(sizes, kinds):
            ts.append(base[k][at[k]:at[k] + m])
            at[k] += m
    else:
        ts = [torch.empty(m, dtype=k, device="cuda").normal_(0.0, std, generator=gen)
              for m, k in zip(sizes, kinds)]
    s = {"kind": case["kind"], "case": case, "ts": ts}
    if case["kind"] == "clip":
        s["out"] = torch.empty(n, dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16,
                               device="cuda")
    if own:  # the list of gradients that a training loop keeps
        from paper_2609_36662_gb300 import aloco as A
        s["list"] = A.GradList(ts)
    return s


# ---------------------------------------------------------------------- run

def run(s):
    if own:
        return _own(s)
    return {"logp": _plain_logp, "policy": _plain_policy, "pref": _plain_pref,
            "norm": _plain_norm, "clip": _plain_clip}[s["kind"]](s)


def _own(s):
    from paper_2609_36662_gb300 import aloco as A
    temp = s["case"].get("temp")
    if s["kind"] == "logp":
        return A.token_logprobs(s["x"], s["t"], temperature=temp)
    if s["kind"] == "policy":
        r = A.policy_loss(s["x"], s["t"], s["adv"], s["old"], s["w"], ref_logp=s["ref"],
                          clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL, temperature=temp)
        return {"terms": r.terms, "logp": r.logp, "grad": r.grad}
    if s["kind"] == "pref":
        r = A.preference_loss(s["x"], s["t"], s["cu"], s["ref"], beta=BETA,
                              label_smoothing=SMOOTH, temperature=temp)
        return {"loss": r.loss, "log_ratios": r.log_ratios, "logp": r.logp, "grad": r.grad}
    if s["kind"] == "norm":
        return A.grad_norm(s["list"])
    return {"norm": A.clip_grads(s["list"], MAX_NORM, out=s["out"]), "out": s["out"]}


def _softmax(s):
    """Probabilities, the tokens' log-probabilities and which rows count."""
    x = s["x"].float() / s["case"]["temp"]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    at = s["t"].clamp(min=0).unsqueeze(-1)
    lp = (x.gather(-1, at) - m - torch.log(z)).squeeze(-1)
    return e / z, lp, at


def _plain_logp(s):
    _, lp, _ = _softmax(s)
    return torch.where(s["t"] >= 0, lp, 0.0)


def _by_logits(s, p, at, live, coef):
    """coef d logp / d logits, row by row, and zeros in the rows that do not
    count."""
    k = (coef / s["case"]["temp"]).unsqueeze(-1)
    g = (p * -k).scatter_add(-1, at, k)
    return torch.where(live.unsqueeze(-1), g, 0.0).to(s["x"].dtype)


def _plain_policy(s):
    p, lp, at = _softmax(s)
    live = s["w"] != 0
    r = torch.exp(lp - s["old"])
    free = r * s["adv"]
    bound = r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * s["adv"]
    d = s["ref"] - lp
    back = torch.exp(d)
    act = free <= bound
    gain, kl = -torch.minimum(free, bound), back - d - 1
    cut = (~act).float()
    coef = s["w"] * (KL * (1 - back) - torch.where(act, free, 0.0))
    terms = torch.stack([torch.where(live, s["w"] * q, 0.0).sum()
                         for q in (gain + KL * kl, gain, kl, cut)])
    return {"terms": terms, "logp": torch.where(live, lp, 0.0),
            "grad": _by_logits(s, p, at, live, coef)}


def _plain_pref(s):
    p, lp, at = _softmax(s)
    live = s["t"] >= 0
    d = torch.where(live, lp - s["ref"], 0.0)
    seqs = torch.arange(s["cu"].numel() - 1, device="cuda").unsqueeze(-1)
    ratios = torch.where(s["seq"] == seqs, d, 0.0).sum(-1)
    z = BETA * (ratios[0::2] - ratios[1::2])
    # -log sigmoid(z) = log(1 + exp(-z)), without overflow
    tail = torch.log1p(torch.exp(-z.abs()))
    loss = (1 - SMOOTH) * (tail + (-z).clamp(min=0)) + SMOOTH * (tail + z.clamp(min=0))
    slope = (torch.sigmoid(z) - (1 - SMOOTH)) * BETA / z.numel()
    coef = torch.stack([slope, -slope], -1).reshape(-1)[s["seq"]]
    return {"loss": loss.mean(), "log_ratios": ratios, "logp": torch.where(live, lp, 0.0),
            "grad": _by_logits(s, p, at, live, coef)}


def _plain_norm(s):
    return torch.sqrt(sum([torch.square(t.float()).sum() for t in s["ts"]]))


def _plain_clip(s):
    norm = _plain_norm(s)
    c = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    flat = torch.cat([t.float() for t in s["ts"]])
    s["out"].copy_(flat * c)
    return {"norm": norm, "out": s["out"]}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions, in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] in ("norm", "clip"):
        flat = torch.cat([t.double() for t in s["ts"]])
        norm = float(torch.dot(flat, flat)) ** 0.5
        out = torch.tensor(norm, dtype=torch.float64)
        if case["kind"] == "norm":
            return out
        return {"norm": out, "out": flat * min(1.0, MAX_NORM / (norm + 1e-6))}
    v = case["v"]
    x = s["x"].reshape(-1, v)
    t = s["t"].reshape(-1)
    live = (s["w"].reshape(-1) > 0) if case["kind"] == "policy" else (t >= 0)
    rows = torch.nonzero(live).reshape(-1)
    lp = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(lp)
    for r in rows.split(512):
        y = x[r].double() / case["temp"]
        lse[r] = torch.logsumexp(y, -1)
        lp[r] = y[torch.arange(len(r), device="cuda"), t[r]] - lse[r]
    shape = s["t"].shape
    if case["kind"] == "logp":
        return lp.reshape(shape)
    if case["kind"] == "policy":
        w, adv, old, ref = (s[k].reshape(-1).double() for k in ("w", "adv", "old", "ref"))
        ratio = (lp - old).exp()
        over = torch.where(adv >= 0, ratio > 1 + CLIP_HIGH, ratio < 1 - CLIP_LOW) & (adv != 0)
        edge = torch.where(adv >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW)
        gain = -adv * torch.where(over, edge, ratio)
        kl = torch.expm1(ref - lp) - (ref - lp)
        mean = [(w * q)[live].sum() for q in (gain + KL * kl, gain, kl, over.double())]
        coef = w * (torch.where(over, 0.0, -adv * ratio) - KL * torch.expm1(ref - lp))
        out = {"terms": torch.stack(mean), "logp": lp.reshape(shape)}
    else:
        lens = _lens(case)
        d = torch.where(live, lp - s["ref"].double(), 0.0)
        ratios = torch.stack([q.sum() for q in d.split(lens)])
        z = BETA * (ratios[0::2] - ratios[1::2])
        near = torch.nn.functional.logsigmoid
        loss = -((1 - SMOOTH) * near(z) + SMOOTH * near(-z)).mean()
        slope = BETA / case["pairs"] * (SMOOTH * torch.sigmoid(z) -
                                        (1 - SMOOTH) * torch.sigmoid(-z))
        each = torch.stack([slope, -slope], 1).reshape(-1).tolist()
        coef = torch.cat([torch.full((n,), k, dtype=torch.float64, device="cuda")
                          for n, k in zip(lens, each)])
        out = {"loss": loss, "log_ratios": ratios, "logp": lp}
    grad = torch.zeros(t.numel(), v, dtype=torch.float64, device="cuda")
    for r in rows.split(512):
        y = torch.exp(x[r].double() / case["temp"] - lse[r, None]).neg_()
        y[torch.arange(len(r), device="cuda"), t[r]] += 1.0
        grad[r] = y * (coef[r, None] / case["temp"])
    out["grad"] = grad.reshape(s["x"].shape)
    return out
