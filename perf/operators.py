"""Cases, plain forms and float64 definitions of the operators around the vocabulary-projection head.

Four operators: layer norm (forward, and a training pass that also returns the gradients), the clipped policy loss with a
KL term, the preference loss over paired sequences, and the Muon update with its orthogonalisation alone.  ``run`` computes
them in elementary torch operations in 32 bits, or, where ``own`` is true, through this repository's entry points.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
COEFFS = (3.4445, -4.7750, 2.0315)
STEPS = 5
LN_EPS = 1e-5
MUON_EPS = 1e-7
MU, LR, DECAY = 0.95, 3e-4, 0.1
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
BETA, SMOOTHING, MARGIN = 0.1, 0.05, 0.25


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the final norm of one token while text is generated: launch latency
        {"name": "ln_one_token", "op": "layer_norm", "rows": 1, "d": 2880, "dtype": "bf16", "wdtype": "bf16", "train": False},
        # the final norm before the head on the 120B-shaped workload, forward and backward
        {"name": "ln_train_120b", "op": "layer_norm", "rows": 16384, "d": 2880, "dtype": "bf16", "wdtype": "bf16", "train": True},
        # the same on the 667B-shaped workload with fp32 norm weights; the largest
        {"name": "ln_train_667b", "op": "layer_norm", "rows": 65536, "d": 7168, "dtype": "bf16", "wdtype": "fp32", "train": True},
        # an odd width and row count in fp32: rows that start off every vector boundary
        {"name": "ln_train_odd", "op": "layer_norm", "rows": 4093, "d": 1111, "dtype": "fp32", "wdtype": "fp32", "train": True},
        # a micro-batch of short answers: one group of samples for one prompt, a scalar advantage each
        {"name": "policy_micro", "op": "policy", "seqs": 8, "tokens": 1021, "aggregate": "token_mean", "kl": 0.0, "adv_per_token": False},
        # a whole rollout batch of long answers with a KL term, the long-context token count
        {"name": "policy_rollout", "op": "policy", "seqs": 256, "tokens": 1048576, "aggregate": "seq_mean", "kl": 0.04, "adv_per_token": True},
        # a few short preference pairs
        {"name": "preference_micro", "op": "preference", "pairs": 4, "tokens": 2047, "kind": "sigmoid", "average": False},
        # many long ragged pairs
        {"name": "preference_long", "op": "preference", "pairs": 128, "tokens": 1048576, "kind": "ipo", "average": True},
        # one small matrix (the tiny workload's width): latency of the chain of products
        {"name": "muon_small", "op": "muon_step", "batch": 1, "rows": 256, "cols": 256, "dtype": "fp32"},
        # four square projections of the 120B-shaped width in one call
        {"name": "muon_square_120b", "op": "muon_step", "batch": 4, "rows": 2880, "cols": 2880, "dtype": "bf16"},
        # tall odd-sized matrices
        {"name": "muon_tall_odd", "op": "muon_step", "batch": 3, "rows": 1999, "cols": 501, "dtype": "fp32"},
        # orthogonalisation alone of wide matrices (mid workload's width by the 667B-shaped width)
        {"name": "muon_orth_wide", "op": "muon_orth", "batch": 2, "rows": 2048, "cols": 7168, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["layer_norm", "policy", "preference", "muon_step", "muon_orth"])
    if op == "layer_norm":
        d = _log_int(rng, 32, 12288)
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rows = min(_log_int(rng, 1, 65536), 65536 * 7168 // (d * (2 if dtype == "fp32" else 1)))
        return {"op": op, "rows": rows, "d": d, "dtype": dtype, "wdtype": rng.choice([dtype, "fp32"]), "train": rng.random() < 0.6}
    if op == "policy":
        seqs = _log_int(rng, 1, 512)
        tokens = min(1048576, seqs * _log_int(rng, 16, 8192) + rng.randrange(64))
        return {"op": op, "seqs": seqs, "tokens": tokens, "aggregate": rng.choice(["token_mean", "seq_mean"]),
                "kl": rng.choice([0.0, 0.001, 0.04]), "adv_per_token": rng.random() < 0.5}
    if op == "preference":
        pairs = _log_int(rng, 1, 256)
        tokens = min(1048576, 2 * pairs * _log_int(rng, 16, 8192) + rng.randrange(64))
        return {"op": op, "pairs": pairs, "tokens": tokens, "kind": rng.choice(["sigmoid", "ipo"]), "average": rng.random() < 0.5}
    rows, cols, batch = _log_int(rng, 48, 4096), _log_int(rng, 48, 4096), _log_int(rng, 1, 16)
    most = 4 * 2880 ** 3 * 4
    m, n = min(rows, cols), max(rows, cols)
    batch = max(1, min(batch, most // (3 * m * m * n + m ** 3)))
    return {"op": op, "batch": batch, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "fp32"] if op == "muon_step" else ["bf16", "fp16"])}


def work(case):
    op = case["op"]
    if op == "layer_norm":
        n, e, we = case["rows"] * case["d"], _size(case["dtype"]), _size(case["wdtype"])
        if case["train"]:
            return {"bytes": 4 * n * e + 4 * case["d"] * we, "flops": 20 * n}
        return {"bytes": 2 * n * e + 2 * case["d"] * we, "flops": 8 * n}
    if op == "policy":
        t = case["tokens"]
        read = 8 + 1 + (4 if case["kl"] else 0) + (4 if case["adv_per_token"] else 0)
        return {"bytes": t * (read + 4), "flops": 20 * t}
    if op == "preference":
        return {"bytes": case["tokens"] * (8 + 1 + 4), "flops": 4 * case["tokens"]}
    m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    flops = case["batch"] * STEPS * (3 * m * m * n + m ** 3)  # the two symmetric products counted once
    per = 2 * _size(case["dtype"]) if op == "muon_orth" else _size(case["dtype"]) + 4 * 4 + 2
    return {"bytes": case["batch"] * m * n * per, "flops": flops}


def _size(name):
    return 4 if name == "fp32" else 2


# ------------------------------------------------------------------------------------------------ inputs
def _ragged(gen, count, tokens):
    """Offsets of `count` sequences that share `tokens` tokens unevenly."""
    w = torch.exp(0.6 * torch.randn(count, generator=gen, dtype=torch.float64))
    cuts = torch.round(torch.cumsum(w, 0) / w.sum() * tokens).to(torch.int64)
    cuts[-1] = tokens
    return torch.cat([torch.zeros(1, dtype=torch.int64), cuts])


def _response_mask(gen, offsets, tokens):
    """True on the answer's tokens: a sequence begins with its prompt, and a few sequences have no answer at all."""
    n = offsets.numel() - 1
    lens = offsets[1:] - offsets[:-1]
    prompt = (lens * torch.rand(n, generator=gen, dtype=torch.float64) * 0.5).to(torch.int64)
    prompt = torch.where(torch.rand(n, generator=gen) < 0.05, lens, prompt)
    seq = torch.repeat_interleave(torch.arange(n), lens)
    return torch.arange(tokens) - offsets[seq] >= prompt[seq]


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": case}
    if op == "layer_norm":
        dt, wdt, d = DT[case["dtype"]], DT[case["wdtype"]], case["d"]
        # hidden states: channels of different size around their own means
        s["x"] = randn(case["rows"], d, dtype=dt).mul_(torch.exp(0.3 * randn(d)).to(dt)).add_((0.5 * randn(d)).to(dt))
        s["w"], s["b"] = (1 + 0.2 * randn(d)).to(wdt), (0.1 * randn(d)).to(wdt)
        if case["train"]:
            s["dy"] = randn(case["rows"], d, dtype=dt)
        return s
    if op in ("policy", "preference"):
        tokens = case["tokens"]
        n = case["seqs"] if op == "policy" else 2 * case["pairs"]
        offsets = _ragged(cpu, n, tokens)
        s["mask"] = _response_mask(cpu, offsets, tokens).cuda()
        s["offsets"] = offsets.cuda()
        s["max_len"] = int((offsets[1:] - offsets[:-1]).max())
        s["logp"] = -torch.nn.functional.softplus(1.5 * randn(tokens) - 0.5)  # log probabilities, mostly near 0
        s["ref"] = (s["logp"] + 0.05 * randn(tokens)).clamp_(max=0.0)
        if op == "policy":
            s["old"] = (s["logp"] + 0.15 * randn(tokens)).clamp_(max=0.0)
            s["adv"] = randn(tokens) if case["adv_per_token"] else randn(n)
            if not case["kl"]:
                s["ref"] = None
        return s
    shape = (case["batch"], case["rows"], case["cols"])
    dt = DT[case["dtype"]]
    # a gradient: a few strong directions over noise
    k = 4
    g = 0.3 * torch.matmul(randn(shape[0], shape[1], k), randn(shape[0], k, shape[2])).add_(randn(*shape))
    s["grad"] = (1e-3 * g).to(dt)
    if op == "muon_step":
        s["p"], s["m"] = 0.02 * randn(*shape), 2e-3 * randn(*shape)
        s["w"] = s["p"].to(torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    return {"layer_norm": _layer_norm, "policy": _policy, "preference": _preference, "muon_step": _muon_step, "muon_orth": _muon_orth}[op](s, case)


def _layer_norm(s, case):
    x, w, b = s["x"], s["w"], s["b"]
    if own:
        import paper_2609_14306_b200 as vp
        y = torch.empty_like(x)
        mean = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
        vp.vp_ln_forward(x, w, b, LN_EPS, y, mean, rstd)
        if not case["train"]:
            return {"y": y}
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        ws = torch.empty(vp.vp_ln_workspace_bytes(*x.shape), dtype=torch.uint8, device=x.device)
        vp.vp_ln_backward(s["dy"], x, w, mean, rstd, dx, dw, db, ws)
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    xf, wf, bf = x.float(), w.float(), b.float()
    xc = xf - xf.mean(1, keepdim=True)
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + LN_EPS)
    xh = xc * rstd
    y = (xh * wf + bf).to(x.dtype)
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].float()
    a = dy * wf
    dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    return {"y": y, "dx": dx.to(x.dtype), "dw": (dy * xh).sum(0).to(w.dtype), "db": dy.sum(0).to(b.dtype)}


def _seq_ids(offsets, tokens):
    return torch.searchsorted(offsets[1:].contiguous(), torch.arange(tokens, device=offsets.device), right=True)


def _seq_sums(v, offsets, max_len):
    """Sums of the token values `v` over each sequence: the sequences laid out as rows of one matrix."""
    at = offsets[:-1, None] + torch.arange(max_len, device=v.device)
    inside = at < offsets[1:, None]
    return torch.where(inside, v[at.clamp(max=v.numel() - 1)], torch.zeros((), device=v.device)).sum(1)


def _policy(s, case):
    logp, old, ref, adv, mask, offsets = s["logp"], s["old"], s["ref"], s["adv"], s["mask"], s["offsets"]
    tokens, kl_coef = case["tokens"], case["kl"]
    if own:
        import paper_2609_14306_b200 as vp
        stats = torch.empty(4, dtype=torch.float32, device=logp.device)
        dlogp = torch.empty_like(logp)
        ws = torch.empty(vp.vp_policy_loss_workspace_bytes(tokens, case["seqs"]), dtype=torch.uint8, device=logp.device)
        vp.vp_policy_loss(logp, old, ref, adv, mask, offsets, CLIP_LOW, CLIP_HIGH, kl_coef, case["aggregate"], stats, dlogp, ws)
        return {"stats": stats, "dlogp": dlogp}
    seq = _seq_ids(offsets, tokens)
    a = adv if case["adv_per_token"] else adv[seq]
    zero = torch.zeros((), device=logp.device)
    lo, hi = 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH
    r = torch.exp(logp - old)
    pol = -torch.minimum(r * a, torch.clamp(r, lo, hi) * a)
    clipped = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
    grad = torch.where(clipped, zero, -a * r)
    kl = torch.zeros_like(logp)
    if ref is not None:
        e = torch.exp(ref - logp)
        kl = e - (ref - logp) - 1
        grad = grad + kl_coef * (1 - e)
    per = torch.where(mask, pol + kl_coef * kl, zero)
    count = mask.sum().clamp(min=1).float()
    if case["aggregate"] == "token_mean":
        loss = per.sum() / count
        weight = 1 / count
    else:
        n = _seq_sums(mask.float(), offsets, s["max_len"])
        some = (n > 0).float().sum().clamp(min=1)
        loss = (_seq_sums(per, offsets, s["max_len"]) / n.clamp(min=1)).sum() / some
        weight = (1 / (n.clamp(min=1) * some))[seq]
    over = lambda v: torch.where(mask, v, zero).sum() / count  # noqa: E731
    stats = torch.stack([loss, over(kl), over(clipped.float()), over(r)])
    return {"stats": stats, "dlogp": torch.where(mask, grad * weight, zero)}


def _preference(s, case):
    logp, ref, mask, offsets = s["logp"], s["ref"], s["mask"], s["offsets"]
    pairs, tokens = case["pairs"], case["tokens"]
    if own:
        import paper_2609_14306_b200 as vp
        stats = torch.empty(3, dtype=torch.float32, device=logp.device)
        rewards = torch.empty(2 * pairs, dtype=torch.float32, device=logp.device)
        dlogp = torch.empty_like(logp)
        ws = torch.empty(vp.vp_preference_loss_workspace_bytes(tokens, pairs), dtype=torch.uint8, device=logp.device)
        vp.vp_preference_loss(logp, ref, mask, offsets, BETA, MARGIN, SMOOTHING, case["kind"], case["average"], stats, rewards, dlogp, ws)
        return {"stats": stats, "rewards": rewards, "dlogp": dlogp}
    zero = torch.zeros((), device=logp.device)
    sums = _seq_sums(torch.where(mask, logp - ref, zero), offsets, s["max_len"])
    n = _seq_sums(mask.float(), offsets, s["max_len"]).clamp(min=1)
    if case["average"]:
        sums = sums / n
    diff = sums[:pairs] - sums[pairs:]
    if case["kind"] == "sigmoid":
        z = BETA * diff - MARGIN
        # -log sigmoid(z) = log(1 + e^-z), kept finite for large |z|
        soft = lambda v: torch.clamp(v, min=0) + torch.log1p(torch.exp(-torch.abs(v)))  # noqa: E731
        per = (1 - SMOOTHING) * soft(-z) + SMOOTHING * soft(z)
        slope = BETA * (SMOOTHING - 1 / (1 + torch.exp(z)))
    else:
        per = (diff - 1 / (2 * BETA)) ** 2
        slope = 2 * (diff - 1 / (2 * BETA))
    slope = slope / pairs
    by_seq = torch.cat([slope, -slope])
    if case["average"]:
        by_seq = by_seq / n
    rewards = BETA * sums
    gap = rewards[:pairs] - rewards[pairs:]
    stats = torch.stack([per.mean(), (gap > 0).float().mean(), gap.mean()])
    return {"stats": stats, "rewards": rewards, "dlogp": torch.where(mask, by_seq[_seq_ids(offsets, tokens)], zero)}


def _orthogonal(u):
    """The Newton-Schulz iteration on each matrix of `u` [batch, rows, cols] in 32 bits."""
    a, b, c = COEFFS
    tall = u.shape[1] > u.shape[2]
    x = u.float()
    if tall:
        x = x.transpose(1, 2)
    norm = (x * x).sum((1, 2), keepdim=True).sqrt().clamp(min=MUON_EPS)
    x = x / norm
    for _ in range(STEPS):
        g = torch.matmul(x, x.transpose(1, 2))
        q = b * g + c * torch.matmul(g, g)
        x = a * x + torch.matmul(q, x)
    return x.transpose(1, 2) if tall else x


def _scale(case):
    return 0.2 * math.sqrt(max(case["rows"], case["cols"]))


def _muon_step(s, case):
    p, m, w, g = s["p"], s["m"], s["w"], s["grad"]
    if own:
        import paper_2609_14306_b200 as vp
        ws = torch.empty(vp.muon_workspace_bytes(case["batch"], case["rows"], case["cols"]), dtype=torch.uint8, device=p.device)
        vp.muon_step(p, m, g, w, LR, MU, DECAY, _scale(case), ws, nesterov=True, coeffs=COEFFS, steps=STEPS, eps=MUON_EPS)
        return {"p": p, "m": m, "w": w}
    gf = g.float()
    m.mul_(MU).add_(gf)
    o = _orthogonal(gf + MU * m)
    p.mul_(1 - LR * DECAY).sub_(LR * _scale(case) * o)
    w.copy_(p)
    return {"p": p, "m": m, "w": w}


def _muon_orth(s, case):
    g = s["grad"]
    if own:
        import paper_2609_14306_b200 as vp
        o = torch.empty_like(g)
        ws = torch.empty(vp.muon_workspace_bytes(case["batch"], case["rows"], case["cols"]), dtype=torch.uint8, device=g.device)
        vp.muon_orthogonalize(g, o, ws, coeffs=COEFFS, steps=STEPS, eps=MUON_EPS)
        return {"o": o}
    return {"o": _orthogonal(g).to(g.dtype)}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f64 = torch.float64
    if op == "layer_norm":
        x, w, b = s["x"].to(f64), s["w"].to(f64), s["b"].to(f64)
        var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        xh = (x - mu) / torch.sqrt(var + LN_EPS)
        out = {"y": torch.addcmul(b, xh, w)}
        if case["train"]:
            dy = s["dy"].to(f64)
            # through the projections that the mean and the scale take out of the gradient
            t = dy * w
            t -= (t * xh).mean(1, keepdim=True) * xh
            t -= t.mean(1, keepdim=True)
            out["dx"] = t / torch.sqrt(var + LN_EPS)
            out["dw"] = torch.einsum("ij,ij->j", dy, xh)
            out["db"] = torch.einsum("ij->j", dy)
        return out
    if op == "policy":
        return _policy_exact(s, case)
    if op == "preference":
        return _preference_exact(s, case)
    if op == "muon_orth":
        return {"o": _orthogonal_exact(s["grad"].to(f64))}
    g = s["grad"].to(f64)
    m = MU * s["m"].to(f64) + g
    p = s["p"].to(f64)
    p = p - LR * DECAY * p - LR * _scale(case) * _orthogonal_exact(MU * m + g)
    return {"p": p, "m": m, "w": p}


def _segments(s):
    """Rows of a [sequences, tokens]-free sum: cumulative sums of float64 values, differences at the offsets."""
    offsets = s["offsets"]

    def total(v):
        c = torch.cat([torch.zeros(1, dtype=torch.float64, device=v.device), torch.cumsum(v.to(torch.float64), 0)])
        return c[offsets[1:]] - c[offsets[:-1]]

    return total


def _policy_exact(s, case):
    lp, mask = s["logp"].double(), s["mask"].double()
    lens = s["offsets"].diff()
    rep = lambda v: torch.repeat_interleave(v, lens)  # noqa: E731
    a = s["adv"].double() if case["adv_per_token"] else rep(s["adv"].double())
    r = torch.exp(lp - s["old"].double())
    bounded = torch.where(a > 0, torch.clamp(r, max=1 + CLIP_HIGH), torch.clamp(r, min=1 - CLIP_LOW))
    free = (bounded == r).double()
    kl, dkl = torch.zeros_like(lp), torch.zeros_like(lp)
    if s["ref"] is not None:
        q = s["ref"].double() - lp
        kl, dkl = torch.expm1(q) - q, -torch.expm1(q)
    per = case["kl"] * kl - bounded * a
    count = mask.sum().clamp(min=1)
    total = _segments(s)
    if case["aggregate"] == "token_mean":
        weight = mask / count
    else:
        n = total(mask).round()
        weight = mask * rep(1 / n.clamp(min=1)) / (n > 0).sum().clamp(min=1)
    stats = torch.stack([(weight * per).sum(), (mask * kl).sum() / count, (mask * (1 - free)).sum() / count, (mask * r).sum() / count])
    return {"stats": stats, "dlogp": weight * (case["kl"] * dkl - free * r * a)}


def _preference_exact(s, case):
    mask, pairs = s["mask"].double(), case["pairs"]
    lens = s["offsets"].diff()
    total = _segments(s)
    n = total(mask).round().clamp(min=1) if case["average"] else torch.ones(2 * pairs, dtype=torch.float64, device=mask.device)
    sums = total(mask * (s["logp"].double() - s["ref"].double())) / n
    chosen, rejected = sums.reshape(2, pairs)
    diff = chosen - rejected
    if case["kind"] == "sigmoid":
        z = BETA * diff - MARGIN
        per = torch.logaddexp(torch.zeros_like(z), -z) + SMOOTHING * z
        slope = BETA * (torch.sigmoid(z) - (1 - SMOOTHING))
    else:
        per = diff ** 2 - diff / BETA + 0.25 / BETA ** 2
        slope = 2 * diff - 1 / BETA
    by_seq = torch.stack([slope, -slope]).reshape(-1) / pairs / n
    stats = torch.stack([per.mean(), (diff > 0).double().mean(), BETA * diff.mean()])
    return {"stats": stats, "rewards": BETA * sums, "dlogp": mask * torch.repeat_interleave(by_seq, lens)}


def _orthogonal_exact(u):
    """The iteration is an odd polynomial in the singular values: with X X^T = Q diag(l) Q^T it is Q diag(f(sqrt l) / sqrt l) Q^T X."""
    a, b, c = COEFFS
    tall = u.shape[1] > u.shape[2]
    x = u.mT if tall else u
    x = x / torch.linalg.matrix_norm(x).clamp(min=MUON_EPS)[:, None, None]
    lam, q = torch.linalg.eigh(x @ x.mT)
    lam = lam.clamp(min=0)
    gain = torch.ones_like(lam)
    for _ in range(STEPS):
        step = a + b * lam + c * lam ** 2
        gain, lam = gain * step, lam * step ** 2
    o = q @ (gain[:, :, None] * (q.mT @ x))
    return o.mT if tall else o
