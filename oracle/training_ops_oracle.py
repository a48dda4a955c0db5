"""Float64 CPU oracles of the operators around the head: layer norm, policy loss, preference loss, Muon.

TEST INFRASTRUCTURE ONLY.  Plain statements of the definitions in float64, one row, one sequence, one matrix at a time;
they share no code with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np

MUON_COEFFS = (3.4445, -4.7750, 2.0315)


def layer_norm(x, g, b, eps):
    """y, mean, rstd of rows of x [rows, d]."""
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if g is not None:
        y = y * g
    if b is not None:
        y = y + b
    return y, mean, rstd


def layer_norm_grad(dy, x, g, eps):
    """dx, dg, db."""
    _, mean, rstd = layer_norm(x, None, None, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy if g is None else dy * g
    dx = rstd[:, None] * (a - a.mean(1, keepdims=True) - xh * (a * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _ranges(offsets, T):
    o = [min(max(int(v), 0), T) for v in offsets]
    return [range(o[i], max(o[i], o[i + 1])) for i in range(len(o) - 1)]


def policy_loss(logp, old, ref, adv, per_token, mask, offsets, lo, hi, kl_coef, aggregate):
    """loss, stats, dlogp; tokens that are masked or outside every sequence are never looked at."""
    T = len(logp)
    grads, per, seq_means = np.zeros(T), [], []
    where = []
    kls, clips, rs = [], [], []
    for s, tokens in enumerate(_ranges(offsets, T)):
        mine = []
        for t in tokens:
            if mask is not None and not mask[t]:
                continue
            A = adv[t] if per_token else adv[s]
            r = math.exp(logp[t] - old[t])
            clipped = (A > 0 and r > 1 + hi) or (A < 0 and r < 1 - lo)
            bounded = min(max(r, 1 - lo), 1 + hi)
            loss = -min(r * A, bounded * A)
            grad = 0.0 if clipped else -A * r
            kl = 0.0
            if ref is not None:
                q = ref[t] - logp[t]
                kl = math.expm1(q) - q
                loss += kl_coef * kl
                grad += kl_coef * -math.expm1(q)
            mine.append(loss)
            kls.append(kl); clips.append(float(clipped)); rs.append(r)
            grads[t] = grad
            where.append((t, s))
        per.append(mine)
    n = sum(len(m) for m in per)
    if n == 0:
        return 0.0, np.zeros(4), np.zeros(T)
    if aggregate == "token_mean":
        loss = math.fsum(v for m in per for v in m) / n
        for t, _ in where:
            grads[t] /= n
    else:
        have = sum(1 for m in per if m)
        loss = math.fsum(math.fsum(m) / len(m) for m in per if m) / have
        for t, s in where:
            grads[t] /= len(per[s]) * have
    return loss, np.array([loss, math.fsum(kls) / n, math.fsum(clips) / n, math.fsum(rs) / n]), grads


def preference_loss(logp, ref, mask, offsets, beta, margin, smoothing, kind, average):
    """loss, stats, rewards, dlogp."""
    T = len(logp)
    sums, counts, tokens_of = [], [], []
    for tokens in _ranges(offsets, T):
        mine = [t for t in tokens if mask is None or mask[t]]
        s = math.fsum(logp[t] - (0.0 if ref is None else ref[t]) for t in mine)
        n = max(len(mine), 1) if average else 1
        sums.append(s / n); counts.append(n); tokens_of.append(mine)
    P = len(sums) // 2
    grads = np.zeros(T)
    if P == 0:
        return 0.0, np.zeros(3), np.zeros(0), grads
    total, wins, gap = [], 0, []
    for i in range(P):
        D = sums[i] - sums[P + i]
        if kind == "sigmoid":
            z = beta * D - margin
            neg = math.log1p(math.exp(-abs(z))) + max(-z, 0.0)
            pos = math.log1p(math.exp(-abs(z))) + max(z, 0.0)
            total.append((1 - smoothing) * neg + smoothing * pos)
            sig = 1 / (1 + math.exp(-z)) if z > -700 else 0.0
            slope = beta * ((sig - 1) * (1 - smoothing) + smoothing * sig)
        else:
            total.append((D - 0.5 / beta) ** 2)
            slope = 2 * (D - 0.5 / beta)
        wins += D > 0
        gap.append(beta * D)
        for sign, s in ((1.0, i), (-1.0, P + i)):
            for t in tokens_of[s]:
                grads[t] += sign * slope / P / counts[s]
    loss = math.fsum(total) / P
    return loss, np.array([loss, wins / P, math.fsum(gap) / P]), beta * np.array(sums), grads


def orthogonalize(g, coeffs=None, steps=5, eps=1e-7):
    """The Newton-Schulz iteration on one matrix."""
    x = g.T if g.shape[0] > g.shape[1] else g
    x = x / max(float(np.linalg.norm(x)), eps)
    for k in range(steps):
        a, b, c = MUON_COEFFS if coeffs is None else coeffs[k]
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.T if g.shape[0] > g.shape[1] else x


def muon_step(p, m, g, lr, mu, nesterov, weight_decay, scale, coeffs=None, steps=5, eps=1e-7):
    """p, m after one update of one matrix, and the orthogonalised update."""
    m = mu * m + g
    o = orthogonalize(g + mu * m if nesterov else m, coeffs, steps, eps)
    return p * (1 - lr * weight_decay) - lr * scale * o, m, o
