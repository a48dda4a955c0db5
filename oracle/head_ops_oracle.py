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
