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


def rounded(u, steps=5, eps=1e-7, coefficients=None):
    """The same with X (times 2^8) as a sum of two fp16 values, the products of the
    larger, and A and b A + c A A in fp16 but for their diagonals."""
    coefficients = coefficients or [COEFFICIENTS] * steps
    u = u.double()
    if u.shape[0] > u.shape[1]:
        return rounded(u.T, steps, eps, coefficients).T
    x = 256 * u / (torch.linalg.matrix_norm(u) + eps)
    for a, b, c in coefficients:
        hi = x.half().double()
        x = hi + (x - hi).half().double()
        g = hi @ hi.T / 65536
        d = g.diagonal().float().double()
        g = (g - torch.diag(g.diagonal())).half().double()
        p = b * g + c * (g @ g + (d[:, None] + d) * g)
        lead = (a + b * d + c * d * d + c * (g @ g).diagonal()).float().double()
        p = (p - torch.diag(p.diagonal())).half().double()
        x = lead[:, None] * x + p @ hi
    return x / 256


def allowed(u, **kw):
    """The norm of a factor's error that the roundings explain: one and a half
    times what they make here (the sums' own, of up to a million fp32 terms in
    the products, and other orders come on top: 2^-17 of the norm)."""
    e = exact(u, **kw)
    return e, 1.5 * float((rounded(u, **kw) - e).norm()) + 2.0 ** -17 * float(e.norm())


def momentum_like(m, n, gen, device="cuda"):
    """Strong directions over a broad rest."""
    r = max(1, min(m, n) // 16)
    a = torch.randn(m, r, generator=gen, device=device)
    b = torch.randn(r, n, generator=gen, device=device)
    w = torch.arange(1, r + 1, device=device).pow(-0.7)
    return 1e-3 * ((a * w) @ b + 0.3 * torch.randn(m, n, generator=gen, device=device))
