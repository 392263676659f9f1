"""Token scores with their gradient, and orthogonalised updates, as cases that
can be timed and checked.

Tuning a language model asks more of a row of logits than the log-probability
of one token: its entropy, which a policy's loss is regularised by and its
collapse is seen from, and its best alternatives, which a smaller model is
taught from.  And its matrices may be updated along the orthogonal factor of
their momentum instead of by AdamW.  The calls are

  scores  aloco.token_scores        log-probabilities of given tokens, with the
                                    entropy and the top alternatives
  sgrad   aloco.token_scores_grad   gradient by the logits of all of these
  ortho   aloco.orthogonalize       orthogonal factor of matrices by
                                    Newton-Schulz products
  muon    aloco.muon_step           momentum, orthogonal factor and update of
                                    the matrices of every replica

With `own` false the same results come from elementary torch operations in 32
bits; with `own` true from the package's kernels.
"""
import math

import torch

own = False

# Five steps X <- a X + (b A + c A A) X with A = X X^T.
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
NORM_EPS = 1e-7
MOMENTUM, DECAY = 0.95, 0.1

# Largest work of any case, listed or drawn.
MOST_BYTES, MOST_FLOPS = 1.1e9, 1.1e13


def listed():
    return [
        # One sampled token comes with its five best alternatives: launches
        # and host work.
        {"name": "scores_one", "kind": "scores", "b": 1, "l": 1, "v": 32000, "x": "bf16",
         "temp": 1.0, "shift": 0, "prompt": 0.0, "banned": False, "top": 5},
        # An ordinary worker's batch: eight sequences of 1024 positions, a
        # quarter prompt, the logits a view without each last position.
        {"name": "scores_32k", "kind": "scores", "b": 8, "l": 1023, "v": 32000, "x": "bf16",
         "temp": 1.0, "shift": 1, "prompt": 0.25, "banned": False, "top": 8},
        # A teacher scores four sequences at the fine-tuning model's
        # vocabulary, with the twenty alternatives that its pupil learns from.
        {"name": "scores_128k", "kind": "scores", "b": 4, "l": 1000, "v": 128256, "x": "bf16",
         "temp": 1.0, "shift": 0, "prompt": 0.0, "banned": False, "top": 20},
        # An odd vocabulary in fp32, at a temperature and with banned tokens.
        {"name": "scores_odd", "kind": "scores", "b": 3, "l": 511, "v": 50257, "x": "f32",
         "temp": 0.7, "shift": 0, "prompt": 0.1, "banned": True, "top": 3},
        # The gradient of a loss with an entropy bonus over a worker's batch.
        {"name": "sgrad_32k", "kind": "sgrad", "b": 8, "l": 1023, "v": 32000, "x": "bf16",
         "temp": 1.0, "shift": 1, "prompt": 0.25, "banned": False, "top": 0},
        # A loss over the alternatives' log-probabilities at the odd vocabulary.
        {"name": "sgrad_odd", "kind": "sgrad", "b": 3, "l": 511, "v": 50257, "x": "f32",
         "temp": 0.7, "shift": 0, "prompt": 0.1, "banned": True, "top": 3},
        # The factor of one low-rank adapter: latency.
        {"name": "ortho_adapter", "kind": "ortho", "batch": 1, "m": 2048, "n": 16, "x": "f32"},
        # The attention projections of the 150M set.
        {"name": "ortho_768", "kind": "ortho", "batch": 48, "m": 768, "n": 768, "x": "f32"},
        # One gated projection of the 1.1B set: few tiles and a long axis.
        {"name": "ortho_5632", "kind": "ortho", "batch": 1, "m": 5632, "n": 2048, "x": "bf16"},
        # Four workers that tune two small matrices each: launches.
        {"name": "muon_tiny", "kind": "muon", "set": "tiny", "workers": 4, "x": "f32",
         "g": "f32", "seed": 0},
        # Matrices of odd sizes at odd places of the vector, rows and columns
        # among them.
        {"name": "muon_odd", "kind": "muon", "set": "odd", "workers": 3, "x": "f32",
         "g": "bf16", "seed": 0},
        # Two layers of the 1.1B set on four workers: the largest.
        {"name": "muon_1b", "kind": "muon", "set": "layers", "workers": 4, "x": "bf16",
         "g": "bf16", "seed": 0},
    ]


def draw(rng):
    kind = rng.choice(["scores", "scores", "sgrad", "sgrad", "ortho", "ortho", "muon", "muon"])
    x = rng.choice(["f32", "bf16"])
    if kind in ("scores", "sgrad"):
        c = {"kind": kind, "v": rng.choice([32000, 128256] + [_size(rng, 40, 131072)] * 3), "x": x,
             "temp": rng.choice([1.0, 1.0, 0.7, 1.3]), "prompt": rng.choice([0.0, 0.1, 0.25, 0.5]),
             "banned": rng.random() < 0.5, "top": rng.choice([0, 1, 2, 5, 8, 20, 32]),
             "b": _size(rng, 1, 16), "l": _size(rng, 1, 2048), "shift": rng.choice([0, 1])}
        while work(c)["bytes"] > MOST_BYTES:
            c["l"] = c["l"] * 2 // 3
        return c
    if kind == "ortho":
        c = {"kind": kind, "batch": _size(rng, 1, 64), "m": _size(rng, 1, 6000),
             "n": _size(rng, 1, 6000), "x": x}
        shrink = ("batch", "m", "n")
    else:
        c = {"kind": kind, "set": "drawn", "workers": rng.randint(1, 8), "x": x,
             "g": rng.choice(["f32", "bf16"]), "seed": rng.randrange(1 << 20)}
        shrink = ("workers",)
    for i in range(64):
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            break
        k = shrink[i % len(shrink)]
        c[k] = max(1, c[k] * 2 // 3)
    return c


def _size(rng, lo, hi):
    """Log-uniform; one in three larger sizes is a multiple of 64."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    return n // 64 * 64 if n > 640 and rng.random() < 1 / 3 else n


# ------------------------------------------------------------------- shapes

def _prompt(case):
    """Leading positions of a sequence that take no part."""
    return int(case["l"] * case["prompt"])


def _sizes(case):
    """(rows, columns) of a replica's matrices; a size of 1 column and a few
    rows stands for what lies between them in the vector and is no matrix."""
    if case["set"] == "tiny":
        return [(512, 64), (512, 64)]
    if case["set"] == "layers":
        d, kv, ffn = 2048, 256, 5632
        return [(d, d), (d, kv), (d, kv), (d, d), (d, ffn), (d, ffn), (ffn, d)] * 2
    if case["set"] == "odd":
        return [(1000, 333), (257, 1025), (50, 50), (1, 129), (767, 1), (7, 4099), (641, 640)]
    import random
    rng = random.Random(case["seed"])
    return [(_size(rng, 1, 2048), _size(rng, 1, 2048)) for _ in range(rng.randint(1, 8))]


def _parts(case):
    """(offset, rows, columns) of the matrices, and the vector's length: in an
    odd set every matrix has a vector of five elements before it."""
    gap = 0 if case["set"] in ("tiny", "layers") else 5
    at, parts = 0, []
    for r, c in _sizes(case):
        at += gap
        parts.append((at, r, c))
        at += r * c
    return parts, at + gap


def _products(r, c):
    """Multiplications and additions of the steps: X X^T and A A are symmetric,
    so that half of each is enough."""
    m, n = min(r, c), max(r, c)
    return STEPS * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)


def _lr(case):
    """Tuning in fp32, or training in bf16 with steps that its values see."""
    return 1e-4 if case["x"] == "f32" else 2e-3


def _elt(kind):
    return 4 if kind == "f32" else 2


def work(case):
    if case["kind"] in ("scores", "sgrad"):
        rows = case["b"] * case["l"]
        live = rows - case["b"] * _prompt(case)
        row = case["v"] * _elt(case["x"])
        if case["kind"] == "scores":
            return {"bytes": live * row + rows * (24 + 8 * case["top"]),
                    "flops": 6 * live * case["v"]}
        return {"bytes": live * row + rows * row + live * (32 + 8 * case["top"]),
                "flops": 7 * live * case["v"]}
    if case["kind"] == "ortho":
        n = case["batch"] * case["m"] * case["n"]
        return {"bytes": n * (_elt(case["x"]) + 2),
                "flops": case["batch"] * _products(case["m"], case["n"])}
    parts, _ = _parts(case)
    n = sum(r * c for _, r, c in parts)
    return {"bytes": case["workers"] * n * (2 * _elt(case["x"]) + _elt(case["g"]) + 8),
            "flops": case["workers"] * sum(_products(r, c) for _, r, c in parts)}


# ------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, std, gen):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)


def _uniform(shape, lo, hi, gen):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=gen)


def _type(kind):
    return torch.float32 if kind == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = _gen(seed)
    if case["kind"] == "ortho":
        return {"case": case, "kind": "ortho",
                "x": _momentum_like(case["batch"], case["m"], case["n"], gen).to(_type(case["x"]))}
    if case["kind"] == "muon":
        return _prepare_muon(case, gen)
    b, l, v = case["b"], case["l"], case["v"]
    # Logits spread as a trained model's, with the tokens that were drawn from
    # them well above the rest; in bf16 many of them are equal.
    full = torch.empty(b, l + case["shift"], v, dtype=_type(case["x"]), device="cuda")
    full.normal_(0.0, 2.0, generator=gen)
    if case["banned"]:
        full[..., v // 3:v // 3 + 17] = -math.inf
        full[..., v - v // 50:] = torch.finfo(full.dtype).min
    t = torch.randint(0, v, full.shape[:-1], generator=gen, device="cuda")
    top = math.log(v) + 1.5
    full.scatter_(-1, t.unsqueeze(-1),
                  _uniform(t.shape + (1,), top - 2.5, top + 4.0, gen).to(full.dtype))
    t = t[:, :l].contiguous()
    x = full[:, :l]
    q = _prompt(case)
    t[:, :q] = -1
    k = min(case["top"], v // 2)
    s = {"case": case, "kind": case["kind"], "x": x, "t": t, "top": k}
    if case["kind"] == "sgrad":
        live = torch.nonzero(t >= 0).numel() // 2
        s["d_logp"] = _normal(t.shape, 1.0 / max(1, live), gen)
        s["d_entropy"] = _normal(t.shape, 0.05 / max(1, live), gen)
        s["d_top"] = _normal(t.shape + (k,), 0.3 / max(1, live), gen) if k else None
        # what the call for the scores left
        if own:
            from paper_2609_36662_gb300 import aloco as A
            s["scores"] = A.token_scores(x, t, top=k, temperature=case["temp"])
        else:
            s["scores"] = _plain_scores(s)
    return s


def _momentum_like(batch, m, n, gen):
    """A few strong directions over a broad rest, as the momentum of a matrix
    in a network has them."""
    r = max(1, min(m, n) // 16)
    weight = torch.arange(1, r + 1, device="cuda", dtype=torch.float32).pow(-0.7)
    strong = torch.bmm(_normal((batch, m, r), 1.0, gen) * weight, _normal((batch, r, n), 1.0, gen))
    return (strong + _normal((batch, m, n), 0.3, gen)) * 1e-3


def _prepare_muon(case, gen):
    parts, n = _parts(case)
    s = {"case": case, "kind": "muon", "parts": parts, "x": [], "g": [], "buf": []}
    for _ in range(case["workers"]):
        x, g, buf = _normal(n, 0.02, gen), _normal(n, 1e-3, gen), _normal(n, 1e-3, gen)
        for at, r, c in parts:
            buf[at:at + r * c] = 4.0 * _momentum_like(1, r, c, gen).reshape(-1)
            g[at:at + r * c] = 0.2 * buf[at:at + r * c] + \
                _momentum_like(1, r, c, gen).reshape(-1)
        s["x"].append(x.to(_type(case["x"])))
        s["g"].append(g.to(_type(case["g"])))
        s["buf"].append(buf)
    if own:  # what a training loop keeps
        from paper_2609_36662_gb300 import aloco as A
        s["matrices"] = A.Matrices(parts)
        s["cfg"] = A.muon_cfg(lr=_lr(case), momentum=MOMENTUM, weight_decay=DECAY,
                              coefficients=[COEFFICIENTS] * STEPS, eps=NORM_EPS)
    return s


# ---------------------------------------------------------------------- run

def run(s):
    if own:
        return _own(s)
    return {"scores": _scores_out, "sgrad": _plain_sgrad, "ortho": _plain_ortho,
            "muon": _plain_muon}[s["kind"]](s)


def _own(s):
    from paper_2609_36662_gb300 import aloco as A
    temp = s["case"].get("temp")
    if s["kind"] == "scores":
        r = A.token_scores(s["x"], s["t"], top=s["top"], temperature=temp)
        out = {"logp": r.logp, "entropy": r.entropy}
        if s["top"]:
            out |= {"top_ids": r.top_ids, "top_logp": r.top_logp}
        return out
    if s["kind"] == "sgrad":
        return A.token_scores_grad(s["x"], s["t"], s["scores"], d_logp=s["d_logp"],
                                   d_entropy=s["d_entropy"], d_top=s["d_top"], temperature=temp)
    if s["kind"] == "ortho":
        return A.orthogonalize(s["x"], coefficients=[COEFFICIENTS] * STEPS, eps=NORM_EPS)
    A.muon_step(s["x"], s["g"], s["buf"], s["matrices"], s["cfg"])
    return {"x": s["x"], "buf": s["buf"]}


def _plain_scores(s):
    """Everything that the scores are made of; rows that take no part hold what
    they hold until _scores_out sets them."""
    x = s["x"].float()
    y = x / s["case"]["temp"]
    m = y.amax(-1, keepdim=True)
    d = y - m
    e = torch.exp(d)
    z = e.sum(-1, keepdim=True)
    logz = torch.log(z)
    p = e / z
    at = s["t"].clamp(min=0).unsqueeze(-1)
    entropy = logz.squeeze(-1) - torch.where(p > 0, p * d, 0.0).sum(-1)
    return {"p": p, "lp": d - logz, "entropy": entropy, "at": at, "top": _best(x, s["top"])}


def _best(x, k):
    """Indices of the k largest of every row, ties by the lowest index."""
    if not k:
        return None
    x = x.clone()
    ids = torch.arange(x.shape[-1], device=x.device, dtype=torch.int32)
    taken = torch.zeros((), device=x.device, dtype=torch.bool)
    found = []
    for _ in range(k):
        open_ = x == torch.where(taken, -math.inf, x).amax(-1, keepdim=True)
        i = torch.where(open_ & ~taken, ids, x.shape[-1]).amin(-1, keepdim=True)
        found.append(i)
        taken = taken | (ids == i)
    return torch.cat(found, -1).long()


def _scores_out(s):
    r = _plain_scores(s)
    live = s["t"] >= 0
    out = {"logp": torch.where(live, r["lp"].gather(-1, r["at"]).squeeze(-1), 0.0),
           "entropy": torch.where(live, r["entropy"], 0.0)}
    if s["top"]:
        out["top_ids"] = torch.where(live.unsqueeze(-1), r["top"], -1).int()
        out["top_logp"] = torch.where(live.unsqueeze(-1), r["lp"].gather(-1, r["top"]), 0.0)
    return out


def _plain_sgrad(s):
    r = _plain_scores(s | {"top": 0})
    ids = s["scores"]["top"]
    total = s["d_logp"] if ids is None else s["d_logp"] + s["d_top"].sum(-1)
    g = -r["p"] * total.unsqueeze(-1)
    g = g - s["d_entropy"].unsqueeze(-1) * \
        torch.where(r["p"] > 0, r["p"] * (r["lp"] + r["entropy"].unsqueeze(-1)), 0.0)
    g = g.scatter_add(-1, r["at"], s["d_logp"].unsqueeze(-1))
    if ids is not None:
        g = g.scatter_add(-1, ids, s["d_top"])
    g = g / s["case"]["temp"]
    return torch.where((s["t"] >= 0).unsqueeze(-1), g, 0.0).to(s["x"].dtype)


def _steps(u):
    """The orthogonal factor of fp32 matrices [..., m, n]."""
    tall = u.shape[-2] > u.shape[-1]
    x = u.mT if tall else u
    a, b, c = COEFFICIENTS
    # (squares of small values do not fit a float: the norm of what the largest leaves)
    top = x.abs().amax((-2, -1), keepdim=True).clamp(min=1e-38)
    x = x / (torch.sqrt(torch.square(x / top).sum((-2, -1), keepdim=True)) * top + NORM_EPS)
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _plain_ortho(s):
    return _steps(s["x"].float()).to(torch.bfloat16).contiguous()


def _plain_muon(s):
    lr = _lr(s["case"])
    for x, g, buf in zip(s["x"], s["g"], s["buf"]):
        for at, r, c in s["parts"]:
            cut = slice(at, at + r * c)
            grad = g[cut].float()
            b = MOMENTUM * buf[cut] + grad
            buf[cut] = b
            o = _steps((grad + MOMENTUM * b).view(r, c)).reshape(-1)
            step = lr * 0.2 * math.sqrt(max(r, c))
            x[cut] = (x[cut].float() * (1 - lr * DECAY) - step * o).to(x.dtype)
    return {"x": s["x"], "buf": s["buf"]}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions, in 64 bits."""
    if case["kind"] == "ortho":
        if work(case)["flops"] > 3e12:
            return None
        return torch.stack([_factor(x.double()) for x in prepare(case, seed)["x"]])
    if case["kind"] == "muon":
        return _exact_muon(case, seed)
    s = prepare(case, seed)
    v, temp, k = case["v"], case["temp"], s["top"]
    x, t = s["x"].reshape(-1, v), s["t"].reshape(-1)
    rows = torch.nonzero(t >= 0).reshape(-1)
    out = {"logp": torch.zeros(t.shape, dtype=torch.float64, device="cuda"),
           "entropy": torch.zeros(t.shape, dtype=torch.float64, device="cuda"),
           "top_ids": torch.full((t.numel(), k), -1, dtype=torch.int32, device="cuda"),
           "top_logp": torch.zeros(t.numel(), k, dtype=torch.float64, device="cuda")}
    grad = torch.zeros(t.numel(), v, dtype=torch.float64, device="cuda") \
        if case["kind"] == "sgrad" else None
    for r in rows.split(256):
        each = torch.arange(len(r), device="cuda")
        lp = torch.log_softmax(x[r].double() / temp, -1)
        p = lp.exp()
        plogp = torch.special.entr(p)
        # a stable descending order keeps equal logits by their index
        ids = torch.sort(x[r].float(), stable=True, dim=-1, descending=True)[1][:, :k]
        if grad is None:
            out["logp"][r] = lp[each, t[r]]
            out["entropy"][r] = plogp.sum(-1)
            out["top_ids"][r] = ids.int()
            out["top_logp"][r] = lp.gather(-1, ids)
            continue
        by_lp = torch.zeros_like(lp)      # what multiplies each log-probability
        by_lp[each, t[r]] = s["d_logp"].reshape(-1)[r].double()
        if k:
            by_lp.scatter_add_(-1, ids, s["d_top"].reshape(-1, k)[r].double())
        # dH = -sum (log p + 1) dp, and sum dp = 0
        h = plogp.sum(-1, keepdim=True)
        by_p = s["d_entropy"].reshape(-1)[r].double()[:, None]
        grad[r] = (by_lp - p * by_lp.sum(-1, keepdim=True) + by_p * (plogp - p * h)) / temp
    if grad is not None:
        return grad.reshape(s["x"].shape)
    shape = s["t"].shape
    return {n: y.reshape(shape + y.shape[1:]) for n, y in out.items() if k or n[:3] != "top"}


def _factor(u):
    """The steps on one matrix in 64 bits, on its smaller side."""
    if u.shape[0] > u.shape[1]:
        return _factor(u.T).T
    x = u / (torch.linalg.matrix_norm(u) + NORM_EPS)
    a, b, c = COEFFICIENTS
    one = torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
    for _ in range(STEPS):
        gram = x @ x.T
        x = (a * one + gram @ (b * one + c * gram)) @ x
    return x


def _exact_muon(case, seed):
    """Of the first worker alone: products in 64 bits are slow."""
    s = prepare(case, seed)
    out = {"x": [None] * case["workers"], "buf": [None] * case["workers"]}
    if work(case)["flops"] / case["workers"] > 5e12:
        return None
    lr = _lr(case)
    x, g, buf = (s[k][0].double() for k in ("x", "g", "buf"))
    for at, r, c in s["parts"]:
        i = torch.arange(at, at + r * c, device="cuda")
        buf[i] = buf[i] * MOMENTUM + g[i]
        u = g[i] + MOMENTUM * buf[i]
        x[i] -= lr * (DECAY * x[i] + 0.2 * max(r, c) ** 0.5 * _factor(u.view(r, c)).reshape(-1))
    out["x"][0], out["buf"][0] = x, buf
    return out
