"""Orthogonal factors stated in 64 bits, and the same with the roundings that the
kernels document: what a kernel may be off follows from these, not from what it
returned."""
import torch

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def exact(u, steps=5, eps=1e-7, coefficients=None):
    """The factor of one matrix."""
    coefficients = coefficients or [COEFFICIENTS] * steps
    u = u.double()
    if u.shape[0] > u.shape[1]:
        return exact(u.T, steps, eps, coefficients).T
    x = u / (torch.linalg.matrix_norm(u) + eps)
    for a, b, c in coefficients:
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def rounded(u, steps=5, eps=1e-7, coefficients=None, shifted=False):
    """The same with X (times 2^8) as a sum of two fp16 values, the products of the
    larger, and A and b A + c A A in fp16 but for their diagonals.  `shifted`: the
    polynomial as c (A + e)^2 - c e^2 with e = b / 2c, where that is not large."""
    coefficients = coefficients or [COEFFICIENTS] * steps
    u = u.double()
    if u.shape[0] > u.shape[1]:
        return rounded(u.T, steps, eps, coefficients, shifted).T
    x = 256 * u / (torch.linalg.matrix_norm(u) + eps)
    for a, b, c in coefficients:
        hi = x.half().double()
        x = hi + (x - hi).half().double()
        g = hi @ hi.T / 65536
        d = g.diagonal().float().double()
        if shifted and abs(b) <= 4 * abs(c):
            e = b / (2 * c)
            g = (g + e * torch.eye(len(d), dtype=g.dtype, device=g.device)).half().double()
            p = c * (g @ g)
            lead = a + b * d + c * (d * d + p.diagonal() / c - g.diagonal() ** 2)
            p = (p - torch.diag(p.diagonal())).half().double()
            x = lead[:, None] * x + p @ hi
            continue
        g = (g - torch.diag(g.diagonal())).half().double()
        p = b * g + c * (g @ g + (d[:, None] + d) * g)
        lead = (a + b * d + c * d * d + c * (g @ g).diagonal()).float().double()
        p = (p - torch.diag(p.diagonal())).half().double()
        x = lead[:, None] * x + p @ hi
    return x / 256


def merged(u, steps=5, eps=1e-7, coefficients=None):
    """The same, two steps at a time where the symmetric matrices alone are multiplied:
    fp16 values with their diagonals, which are right in fp32."""
    coefficients = coefficients or [COEFFICIENTS] * steps
    u = u.double()
    if u.shape[0] > u.shape[1]:
        return merged(u.T, steps, eps, coefficients).T

    def kept(s, d):
        d = d.float().double()
        s = s - torch.diag(s.diagonal()) + torch.diag(d)
        return s.half().double(), d

    def product(p, q):
        (p, dp), (q, dq) = p, q
        s = p @ q
        return kept(s, s.diagonal() - p.diagonal() * q.diagonal() + dp * dq)

    def poly(p, k):
        (p, d), (a, b, c) = p, k
        s = p @ p
        return kept(b * p + c * s, a + b * d + c * (s.diagonal() - p.diagonal() ** 2 + d * d))

    x = 256 * u / (torch.linalg.matrix_norm(u) + eps)
    todo = list(coefficients)
    while todo:
        hi = x.half().double()
        x = hi + (x - hi).half().double()
        g = hi @ hi.T / 65536
        g = kept(g, g.diagonal())
        q = p = poly(g, todo.pop(0))
        if todo:
            g = product(product(p, g), p)
            q = product(poly(g, todo.pop(0)), p)
        x = q[1][:, None] * x + (q[0] - torch.diag(q[0].diagonal())) @ hi
    return x / 256


def allowed(u, two_at_a_time=False, **kw):
    """The norm of a factor's error that the roundings explain: one and a half
    times what they make here (the sums' own, of up to a million fp32 terms in
    the products, and other orders come on top: 2^-17 of the norm)."""
    e = exact(u, **kw)
    # (which form a matrix takes depends on its company)
    forms = [merged(u, **kw)] if two_at_a_time else \
        [rounded(u, shifted=s, **kw) for s in (False, True)]
    return e, 1.5 * max(float((r - e).norm()) for r in forms) + 2.0 ** -17 * float(e.norm())


def momentum_like(m, n, gen, device="cuda"):
    """Strong directions over a broad rest."""
    r = max(1, min(m, n) // 16)
    a = torch.randn(m, r, generator=gen, device=device)
    b = torch.randn(r, n, generator=gen, device=device)
    w = torch.arange(1, r + 1, device=device).pow(-0.7)
    return 1e-3 * ((a * w) @ b + 0.3 * torch.randn(m, n, generator=gen, device=device))
