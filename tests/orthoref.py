"""Newton-Schulz directions and optimiser steps in 64 bits."""
import torch

USUAL = (3.4445, -4.7750, 2.0315)


def direction(u, steps=5, eps=1e-7, coefs=None):
    u = u.double()
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.norm() + eps)
    for i in range(steps):
        a, b, c = USUAL if coefs is None else coefs[i]
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def update(w, momentum, g, mask, lr, mu, nesterov, decay, scale, **kw):
    keep = torch.ones_like(w, dtype=torch.bool) if mask is None else mask != 0
    g, momentum = torch.where(keep, g.double(), 0.0), torch.where(keep, momentum.double(), 0.0)
    momentum = mu * momentum + g
    o = direction(g + mu * momentum if nesterov else momentum, **kw)
    return torch.where(keep, (1 - lr * decay) * w.double() - lr * scale * o, 0.0), momentum, o


def matrix(kind, m, k, seed, device="cpu"):
    """A matrix to orthogonalise: noise, or directions that fall off (their inverse condition down to 1e-6)."""
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(m, k, generator=gen, dtype=torch.float64)
    if kind != "noise":
        n = min(m, k)
        u, _, v = torch.linalg.svd(g, full_matrices=False)
        s = 1.0 / torch.arange(1, n + 1, dtype=torch.float64) ** {"falling": 1, "steep": 2}[kind]
        g = (u * s) @ v
    return g.to(device)
