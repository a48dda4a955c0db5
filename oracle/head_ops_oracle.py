"""Float64 definitions of the operators from the residual stream to log probabilities (test infrastructure only).

Written from the formulas, in torch on whatever device the inputs are on; inputs are taken as the exact values of their type.
"""
from __future__ import annotations

import torch

F64 = torch.float64
BLOCK = 128


def rms_norm(z, g, eps):
    """(y, rstd) of rows z: y = z g / sqrt(mean(z^2) + eps)."""
    z = z.to(F64)
    rstd = 1 / torch.sqrt((z * z).mean(1) + eps)
    y = z * rstd[:, None]
    return (y if g is None else y * g.to(F64)), rstd


def rms_norm_grad(dy, dz, z, g, eps):
    """(dx, dg) for upstream gradients dy of y and dz of z (or None)."""
    dy, z = dy.to(F64), z.to(F64)
    _, rstd = rms_norm(z, None, eps)
    zh = z * rstd[:, None]
    a = dy if g is None else dy * g.to(F64)
    dx = rstd[:, None] * (a - zh * (a * zh).mean(1, keepdim=True))
    return (dx if dz is None else dx + dz.to(F64)), (dy * zh).sum(0)


def group_scales(y):
    """Scale of each 128 columns of rows y: max|y| / 448, 1 where that is 0."""
    m = torch.stack([p.abs().amax(1) for p in torch.split(y.to(F64), BLOCK, dim=1)], 1)
    return torch.where(m > 0, m / 448, torch.ones_like(m))


def spread_columns(scales, d):
    """A row's scales as one for each of its d columns."""
    return torch.repeat_interleave(scales.to(F64), BLOCK, dim=1)[:, :d]


def block_scales(w):
    """Scale of each 128 x 128 block of w: max|w| / 448, 1 where that is 0."""
    m = torch.stack([torch.stack([p.abs().max() for p in torch.split(r, BLOCK, dim=1)]) for r in torch.split(w.to(F64), BLOCK, dim=0)])
    return torch.where(m > 0, m / 448, torch.ones_like(m))


def spread_blocks(scales, rows, d):
    """Blocks' scales as one for each element of a [rows, d] weight."""
    return torch.repeat_interleave(spread_columns(scales, d), BLOCK, dim=0)[:rows]


def token_logp(h, w, tokens, temperature, ignore_index=-100):
    """dict of logits (before the temperature), lse, entropy and logp of given tokens (0 where ignored or outside the vocabulary)."""
    x = h.to(F64) @ w.to(F64).mT
    logq = torch.log_softmax(x / temperature, dim=1)
    p = torch.exp(logq)
    out = {"x": x, "lse": torch.logsumexp(x / temperature, dim=1), "entropy": -(p * logq).sum(1), "logq": logq}
    if tokens is not None:
        t = tokens.long()
        valid = (t != ignore_index) & (t >= 0) & (t < w.shape[0])
        out["valid"] = valid
        out["logp"] = torch.where(valid, logq.gather(1, t.clamp(0, w.shape[0] - 1)[:, None])[:, 0], torch.zeros((), dtype=F64, device=h.device))
    return out


def token_logp_grad(h, w, tokens, dlogp, dent, temperature, ignore_index=-100):
    """(dH, dW, G): gradients for upstream gradients dlogp and dent (either may be None), and that of the logits."""
    o = token_logp(h, w, tokens, temperature, ignore_index)
    p = torch.exp(o["logq"])
    g = torch.zeros_like(p)
    if dlogp is not None:
        u = torch.where(o["valid"], dlogp.to(F64), torch.zeros((), dtype=F64, device=h.device))
        g -= p * u[:, None]
        g.scatter_add_(1, tokens.long().clamp(0, w.shape[0] - 1)[:, None], u[:, None])
    if dent is not None:
        g -= dent.to(F64)[:, None] * p * (o["logq"] + o["entropy"][:, None])
    g /= temperature
    return g @ w.to(F64), g.mT @ h.to(F64), g
