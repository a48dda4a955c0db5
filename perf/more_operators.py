"""Cases, plain forms and float64 definitions of the operators from the residual stream to log probabilities.

Four operators: the RMS norm with the residual's addition (forward, a training pass that also returns the gradients, and the
output in 8 bits with a scale for each 128 columns), log probabilities of given tokens with entropy and top alternatives (forward,
and a training pass), the same from 8-bit operands with block scales, and the quantisation of a weight into such blocks.
``run`` computes them in elementary torch operations in 32 bits, or, where ``own`` is true, through this repository's entry points.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
BLOCK = 128
EPS = 1e-6
IGNORE = -100
LARGEST = 6 * 8192 * 201088 * 2880  # multiply-adds are counted as two: a training pass's three products, without the recomputed one


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the final norm of one token while text is generated: launch latency
        {"name": "rms_one_token", "op": "rms", "rows": 1, "d": 2880, "dtype": "bf16", "wdtype": "bf16", "residual": True, "train": False},
        # the final norm of the 120B-shaped workload's batch, forward and backward, the residual stream passed on
        {"name": "rms_train_120b", "op": "rms", "rows": 16384, "d": 2880, "dtype": "bf16", "wdtype": "bf16", "residual": True, "train": True},
        # an odd width and row count in fp32, no residual: rows that start off every vector boundary
        {"name": "rms_train_odd", "op": "rms", "rows": 4093, "d": 1111, "dtype": "fp32", "wdtype": "fp32", "residual": False, "train": True},
        # 8-bit activations for the head of the 667B-shaped workload
        {"name": "rms_fp8_667b", "op": "rms_fp8", "rows": 32768, "d": 7168, "dtype": "bf16", "wdtype": "fp32", "residual": True},
        # one new token while text is generated, with its alternatives: one reading of the head's weight
        {"name": "logp_one_token", "op": "logp", "tokens": 1, "d": 2880, "vocab": 201088, "top": 8, "temperature": 1.0, "train": False},
        # a small ragged batch of new tokens on the mid workload's width, an odd vocabulary, sampled at a temperature
        {"name": "logp_small_batch", "op": "logp", "tokens": 61, "d": 2048, "vocab": 32771, "top": 20, "temperature": 0.7, "train": False},
        # scoring a rollout micro-batch on the 120B-shaped workload
        {"name": "logp_score_120b", "op": "logp", "tokens": 4096, "d": 2880, "vocab": 201088, "top": 8, "temperature": 1.0, "train": False},
        # a policy step's log probabilities and entropy bonus with their gradients; the largest
        {"name": "logp_train_120b", "op": "logp", "tokens": 8192, "d": 2880, "vocab": 201088, "top": 0, "temperature": 1.0, "train": True},
        # sixteen sequences being generated with an 8-bit head of the 667B-shaped workload
        {"name": "logp8_decode_667b", "op": "logp8", "tokens": 16, "d": 7168, "vocab": 129280, "top": 8, "temperature": 1.0},
        # a reference model's log probabilities of a rollout batch from its 8-bit head
        {"name": "logp8_score_667b", "op": "logp8", "tokens": 8192, "d": 7168, "vocab": 129280, "top": 0, "temperature": 1.0},
        # a reference model's head made 8-bit after its weights have been renewed
        {"name": "quant_head_120b", "op": "quant", "rows": 201088, "d": 2880, "dtype": "bf16"},
        # a ragged fp32 master weight
        {"name": "quant_odd", "op": "quant", "rows": 1999, "d": 1111, "dtype": "fp32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms", "rms", "rms_fp8", "logp", "logp", "logp8", "quant"])
    if op in ("rms", "rms_fp8"):
        d = _log_int(rng, 32, 12288)
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rows = min(_log_int(rng, 1, 65536), 32768 * 7168 // (d * (2 if dtype == "fp32" else 1)))
        case = {"op": op, "rows": rows, "d": d, "dtype": dtype, "wdtype": rng.choice([dtype, "fp32"]), "residual": rng.random() < 0.7}
        if op == "rms":
            case["train"] = rng.random() < 0.6
        return case
    if op == "quant":
        d = _log_int(rng, 16, 8192)
        return {"op": op, "rows": min(_log_int(rng, 1, 201088), 201088 * 2880 // d), "d": d, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    unit = 8 if op == "logp" else 16
    d = unit * _log_int(rng, 256 // unit, 7168 // unit)
    vocab = _log_int(rng, 1000, 201088)
    train = op == "logp" and rng.random() < 0.4
    tokens = _log_int(rng, 1, 8192)
    tokens = max(1, min(tokens, LARGEST // ((6 if train else 2) * vocab * d)))
    case = {"op": op, "tokens": tokens, "d": d, "vocab": vocab, "top": 0 if train else rng.choice([0, 1, 5, 8, 20]),
            "temperature": rng.choice([1.0, 1.0, 0.7, 1.3])}
    if op == "logp":
        case["train"] = train
    return case


def _size(name):
    return 4 if name == "fp32" else 2


def _groups(n):
    return -(-n // BLOCK)


def work(case):
    op = case["op"]
    if op in ("rms", "rms_fp8"):
        n, e, we, d = case["rows"] * case["d"], _size(case["dtype"]), _size(case["wdtype"]), case["d"]
        arrays = 2 if case["residual"] else 1  # x and the residual; the sum is written where there is one
        if op == "rms_fp8":
            return {"bytes": n * (arrays * e + (e if arrays == 2 else 0) + 1) + 4 * case["rows"] * _groups(d) + d * we, "flops": 10 * n}
        if case["train"]:
            # in: x, residual, dy, dz; out: y, z, dx
            return {"bytes": n * e * (7 if arrays == 2 else 4) + 2 * d * we, "flops": 20 * n}
        return {"bytes": n * e * (4 if arrays == 2 else 2) + d * we, "flops": 6 * n}
    if op == "quant":
        n = case["rows"] * case["d"]
        return {"bytes": n * (_size(case["dtype"]) + 1) + 4 * _groups(case["rows"]) * _groups(case["d"]), "flops": 3 * n}
    t, d, v = case["tokens"], case["d"], case["vocab"]
    out = t * (4 + 4 + 12 * case["top"])
    if op == "logp8":
        return {"bytes": (t + v) * d + 4 * _groups(d) * (t + _groups(v)) + 8 * t + out, "flops": 2 * t * d * v}
    if case["train"]:
        return {"bytes": 2 * (2 * t * d + 2 * v * d) + 16 * t + out, "flops": 6 * t * d * v}
    return {"bytes": 2 * (t + v) * d + 8 * t + out, "flops": 2 * t * d * v}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": case}
    if op in ("rms", "rms_fp8"):
        dt, wdt, d, rows = DT[case["dtype"]], DT[case["wdtype"]], case["d"], case["rows"]
        # a residual stream: channels of different size, a few of them large; a block's output is smaller than the stream
        channel = torch.exp(0.4 * randn(d))
        channel[:: max(1, d // 5)] *= 8
        s["x"] = randn(rows, d, dtype=dt).mul_(channel.to(dt))
        s["r"] = randn(rows, d, dtype=dt).mul_((2 * channel).to(dt)) if case["residual"] else None
        s["w"] = (1 + 0.3 * randn(d)).to(wdt)
        if case.get("train"):
            s["dy"] = randn(rows, d, dtype=dt)
            s["dz"] = randn(rows, d, dtype=dt) if case["residual"] else None
        return s
    if op == "quant":
        # rows of different size: rare tokens have small vectors
        s["w"] = randn(case["rows"], case["d"], dtype=DT[case["dtype"]]).mul_((0.02 * torch.exp(0.5 * randn(case["rows"], 1))).to(DT[case["dtype"]]))
        return s
    t, d, v = case["tokens"], case["d"], case["vocab"]
    # Hidden states of about unit size and weights that give logits a spread of about 2, both on a grid on which every sum of
    # products is exact in 32 bits: which alternative comes first then follows from the definition (ties, which do occur, go to the
    # lowest id) and not from the order of a sum.  Half of the given tokens are likely ones, as a policy's own choices are.
    tokens = torch.randint(0, v, (t,), generator=gen, device="cuda")
    likely = torch.rand(t, generator=gen, device="cuda") < 0.5
    ints = (randn(v, d, dtype=torch.float32 if v * d < 1 << 26 else torch.bfloat16) * 8).round_().clamp_(-16, 16)
    lean = torch.where(likely, 5.0 / math.sqrt(d), 0.0)[:, None] * ints[tokens].float() / 8
    h = ((randn(t, d) + lean) * 4).round_().clamp_(-16, 16)
    unit = 2.0 ** round(math.log2(2.0 / (8 * math.sqrt(d))))
    tokens[torch.rand(t, generator=gen, device="cuda") < 0.05] = IGNORE  # prompt tokens in between
    if op == "logp8":
        # whole numbers up to 16 are e4m3 numbers; scales are powers of two
        pow2 = lambda *shape: 2.0 ** torch.randint(-1, 2, shape, generator=gen, device="cuda").float()  # noqa: E731
        s["h"], s["hs"] = h.to(F8), 0.25 * pow2(t, _groups(d))
        s["w"], s["ws"] = ints.to(F8), unit * pow2(_groups(v), _groups(d))
    else:
        s["h"], s["w"] = (h / 4).to(torch.bfloat16), ints.mul_(unit).to(torch.bfloat16)
        if case["train"]:
            s["dlogp"] = randn(t) / t
            s["dent"] = -0.01 * torch.rand(t, generator=gen, device="cuda") / t
    del ints
    s["tokens"] = tokens.to(torch.int32)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    return {"rms": _rms, "rms_fp8": _rms_fp8, "logp": _logp, "logp8": _logp8, "quant": _quant}[case["op"]](s, case)


def _sum_and_norm(x, r, w):
    z = x if r is None else (x.float() + r.float()).to(x.dtype)
    zf = z.float()
    rstd = torch.rsqrt((zf * zf).mean(1, keepdim=True) + EPS)
    return z, zf * rstd, rstd, w.float()


def _rms(s, case):
    x, r, w = s["x"], s["r"], s["w"]
    if own:
        import paper_2609_14306_b200 as vp
        y = torch.empty_like(x)
        z = x if r is None else torch.empty_like(x)
        rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device) if case["train"] else None
        vp.vp_rms_forward(x, r, w, EPS, y, None if r is None else z, rstd)
        out = {"y": y} if r is None else {"y": y, "z": z}
        if case["train"]:
            dx, dw = torch.empty_like(x), torch.empty_like(w)
            ws = torch.empty(vp.vp_rms_workspace_bytes(*x.shape), dtype=torch.uint8, device=x.device)
            vp.vp_rms_backward(s["dy"], s["dz"], z, w, rstd, dx, dw, ws)
            out.update(dx=dx, dw=dw)
        return out
    z, zh, rstd, wf = _sum_and_norm(x, r, w)
    out = {"y": (zh * wf).to(x.dtype)} if r is None else {"y": (zh * wf).to(x.dtype), "z": z}
    if case["train"]:
        dy = s["dy"].float()
        a = dy * wf
        dx = rstd * (a - zh * (a * zh).mean(1, keepdim=True))
        if r is not None:
            dx = dx + s["dz"].float()
        out.update(dx=dx.to(x.dtype), dw=(dy * zh).sum(0).to(w.dtype))
    return out


def _pad(m, rows, cols):
    """`m` with zeros up to `rows` x `cols`."""
    out = torch.zeros(rows, cols, dtype=m.dtype, device=m.device)
    out[: m.shape[0], : m.shape[1]] = m
    return out


def _to_e4m3(y, amax):
    """(scale, the values nearest to y / scale in 8 bits), amax being each element's group's."""
    scale = torch.where(amax > 0, amax / F8_MAX, torch.ones_like(amax))
    return scale, (y / scale).to(F8)


def _rms_fp8(s, case):
    x, r, w = s["x"], s["r"], s["w"]
    rows, d = x.shape
    if own:
        import paper_2609_14306_b200 as vp
        z = None if r is None else torch.empty_like(x)
        q = torch.empty(rows, d, dtype=F8, device=x.device)
        scales = torch.empty(rows, _groups(d), dtype=torch.float32, device=x.device)
        vp.vp_rms_forward_fp8(x, r, w, EPS, q, scales, z, None)
        return {"q": q, "scales": scales} if r is None else {"q": q, "scales": scales, "z": z}
    z, zh, _, wf = _sum_and_norm(x, r, w)
    y = _pad(zh * wf, rows, _groups(d) * BLOCK).view(rows, -1, BLOCK)
    scale, q = _to_e4m3(y, y.abs().amax(2, keepdim=True))
    out = {"q": q.view(rows, -1)[:, :d].contiguous(), "scales": scale.view(rows, -1)}
    if r is not None:
        out["z"] = z
    return out


def _quant(s, case):
    w = s["w"]
    rows, d = w.shape
    if own:
        import paper_2609_14306_b200 as vp
        q = torch.empty(rows, d, dtype=F8, device=w.device)
        scales = torch.empty(_groups(rows), _groups(d), dtype=torch.float32, device=w.device)
        vp.vp_fp8_quantize_blocks(w, q, scales)
        return {"q": q, "scales": scales}
    y = w.float()
    if rows % BLOCK or d % BLOCK:
        y = _pad(y, _groups(rows) * BLOCK, _groups(d) * BLOCK)
    y = y.view(_groups(rows), BLOCK, _groups(d), BLOCK)
    scale, q = _to_e4m3(y, y.abs().amax((1, 3), keepdim=True))
    return {"q": q.view(_groups(rows) * BLOCK, -1)[:rows, :d].contiguous(), "scales": scale.view(_groups(rows), -1)}


def _top(logits, k):
    """The k largest of each row and their columns, larger first, among equals the lower column."""
    rows = torch.arange(logits.shape[0], device=logits.device)
    left = logits.clone()
    columns = torch.arange(logits.shape[1], device=logits.device)
    vals, ids = [], []
    for _ in range(k):
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, columns, logits.shape[1]).amin(1)
        vals.append(best[:, 0])
        ids.append(at)
        left[rows, at] = -math.inf
    return torch.stack(vals, 1), torch.stack(ids, 1)


def _statistics(logits, tokens, k):
    """Log probability of `tokens` (0 where ignored), entropy, and the alternatives, from a block of logits."""
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    lse = top + torch.log(z)
    entropy = torch.log(z)[:, 0] - ((logits - top) * e).sum(1) / z[:, 0]
    valid = tokens >= 0
    chosen = logits[torch.arange(len(tokens), device=logits.device), tokens.clamp(min=0).long()]
    out = {"logp": torch.where(valid, chosen - lse[:, 0], torch.zeros((), device=logits.device)), "entropy": entropy}
    if k:
        vals, ids = _top(logits, k)
        out["top_logp"], out["top_ids"] = vals - lse, ids.to(torch.int32)
    return out, e / z, lse


def _cat(parts):
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _logp(s, case):
    h, w, tokens, k, temp = s["h"], s["w"], s["tokens"], case["top"], case["temperature"]
    t = case["tokens"]
    if own:
        import paper_2609_14306_b200 as vp
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=h.device)  # noqa: E731
        logp, lse, entropy = f32(t), f32(t), f32(t)
        top_logp = f32(t, k) if k else None
        top_ids = torch.empty(t, k, dtype=torch.int32, device=h.device) if k else None
        ws = torch.empty(vp.vp_token_logp_workspace_bytes(*h.shape, w.shape[0], k), dtype=torch.uint8, device=h.device)
        vp.vp_token_logp_forward(h, w, tokens, temp, IGNORE, logp, lse, entropy, top_logp, top_ids, ws)
        out = {"logp": logp, "entropy": entropy}
        if k:
            out.update(top_logp=top_logp, top_ids=top_ids)
        if case["train"]:
            chunk, block_v = min(16384, -(-t // 128) * 128), 8192
            dh, dw = torch.empty_like(h), f32(*w.shape)
            ws = torch.empty(vp.vp_ce_workspace_bytes(chunk, h.shape[1], block_v), dtype=torch.uint8, device=h.device)
            vp.vp_token_logp_backward(h, w, tokens, lse, entropy, s["dlogp"], s["dent"], temp, IGNORE, dh, dw, block_v, chunk, False, ws)
            out.update(dh=dh, dw=dw.to(w.dtype))
        return out
    wf = w.float()
    parts = []
    dw = torch.zeros(w.shape, dtype=torch.float32, device=w.device) if case["train"] else None
    for i in range(0, t, 2048):
        hf, tok = h[i:i + 2048].float(), tokens[i:i + 2048]
        logits = torch.matmul(hf, wf.t()) / temp
        out, p, lse = _statistics(logits, tok, k)
        if case["train"]:
            valid = tok >= 0
            dlogp = torch.where(valid, s["dlogp"][i:i + 2048], torch.zeros((), device=h.device))[:, None]
            dent = s["dent"][i:i + 2048, None]
            g = -p * (dlogp + dent * ((logits - lse) + out["entropy"][:, None]))
            rows = torch.arange(len(tok), device=h.device)
            g[rows, tok.clamp(min=0).long()] += dlogp[:, 0]
            g = g / temp
            out["dh"] = torch.matmul(g, wf).to(h.dtype)
            dw += torch.matmul(g.t(), hf)
        parts.append(out)
    out = _cat(parts)
    if case["train"]:
        out["dw"] = dw.to(w.dtype)
    return out


def _dequant(q, rows_of, cols_of, dtype):
    """The numbers that q stands for, `rows_of` and `cols_of` being its scales spread over rows, then columns."""
    v = q.to(dtype)
    for c in range(0, q.shape[1], BLOCK):
        v[:, c:c + BLOCK] *= rows_of(cols_of[:, c // BLOCK])[:, None].to(dtype)
    return v


def _weights(s, dtype):
    rows = s["w"].shape[0]
    return _dequant(s["w"], lambda c: torch.repeat_interleave(c, BLOCK)[:rows], s["ws"], dtype)


def _logp8(s, case):
    h, w, tokens, k, temp = s["h"], s["w"], s["tokens"], case["top"], case["temperature"]
    t = case["tokens"]
    if own:
        import paper_2609_14306_b200 as vp
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=h.device)  # noqa: E731
        logp, lse, entropy = f32(t), f32(t), f32(t)
        top_logp = f32(t, k) if k else None
        top_ids = torch.empty(t, k, dtype=torch.int32, device=h.device) if k else None
        ws = torch.empty(vp.vp_token_logp_fp8_workspace_bytes(*h.shape, w.shape[0], k), dtype=torch.uint8, device=h.device)
        vp.vp_token_logp_fp8_forward(h, s["hs"], w, s["ws"], tokens, temp, IGNORE, logp, lse, entropy, top_logp, top_ids, ws)
        out = {"logp": logp, "entropy": entropy}
        if k:
            out.update(top_logp=top_logp, top_ids=top_ids)
        return out
    wf = _weights(s, torch.float32)
    hf = _dequant(h, lambda c: c, s["hs"], torch.float32)
    return _cat([_statistics(torch.matmul(hf[i:i + 2048], wf.t()) / temp, tokens[i:i + 2048], k)[0] for i in range(0, t, 2048)])


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, f64 = case["op"], torch.float64
    if op in ("rms", "rms_fp8"):
        x, w = s["x"].to(f64), s["w"].to(f64)
        out = {}
        if case["residual"]:
            # the norm is of the sum as it is stored
            out["z"] = x.add_(s["r"].to(f64))
            x = x.to(s["x"].dtype).to(f64)
        norm = torch.linalg.vector_norm(x, dim=1, keepdim=True) / math.sqrt(case["d"])
        rms = torch.hypot(norm, torch.full_like(norm, math.sqrt(EPS)))
        if op == "rms":
            out["y"] = x * w / rms
            if case["train"]:
                dy = s["dy"].to(f64)
                unit = x / rms
                out["dw"] = torch.einsum("ij,ij->j", dy, unit)
                t = dy * w
                # the gradient loses its part along the row
                t = (t - unit * torch.einsum("ij,ij->i", t, unit)[:, None] / case["d"]) / rms
                out["dx"] = t + s["dz"].to(f64) if case["residual"] else t
            return out
        y = x * w / rms
        pieces = torch.split(y, BLOCK, dim=1)
        scales = torch.stack([torch.linalg.vector_norm(p, ord=math.inf, dim=1) for p in pieces], 1) / F8_MAX
        out["q"] = torch.cat([p / scales[:, i:i + 1] for i, p in enumerate(pieces)], 1)
        out["scales"] = scales
        return out
    if op == "quant":
        q, scales = [], []
        for rows in torch.split(s["w"], BLOCK, dim=0):
            row = [(p.to(f64), p.to(f64).abs().max() / F8_MAX) for p in torch.split(rows, BLOCK, dim=1)]
            scales.append(torch.stack([c for _, c in row]))
            # numbers of this size need no more than 32 bits to be told from their neighbours in 8
            q.append(torch.cat([p / c for p, c in row], 1).float())
        return {"q": torch.cat(q), "scales": torch.stack(scales)}
    if op == "logp8":
        w, h = _weights(s, f64), _dequant(s["h"], lambda c: c, s["hs"], f64)
    else:
        w, h = s["w"].to(f64), s["h"].to(f64)
    k, temp, tokens = case["top"], case["temperature"], s["tokens"].long()
    parts, dw = [], None
    for i in range(0, case["tokens"], 1024):
        tok = tokens[i:i + 1024]
        valid = tok >= 0
        logq = torch.log_softmax((h[i:i + 1024] @ w.mT) / temp, dim=1)
        out = {"logp": torch.where(valid, logq.gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0)}
        p = torch.exp(logq)
        out["entropy"] = -torch.linalg.vecdot(p, logq)
        if k:
            # a stable order puts the lower column first among equals
            vals, ids = torch.sort(logq, dim=1, descending=True, stable=True)
            out["top_logp"], out["top_ids"] = vals[:, :k].clone(), ids[:, :k].to(torch.int32)
            del vals, ids
        if case.get("train"):
            u = torch.where(valid, s["dlogp"][i:i + 1024].to(f64), 0.0)
            v = s["dent"][i:i + 1024].to(f64)
            g = torch.zeros_like(p).scatter_(1, tok.clamp(min=0)[:, None], u[:, None])
            logq += out["entropy"][:, None]
            g -= p * (u[:, None] + v[:, None] * logq)
            g /= temp
            out["dh"] = g @ w
            part = g.mT @ h[i:i + 1024]
            dw = part if dw is None else dw.add_(part)
        parts.append(out)
    out = _cat(parts)
    if dw is not None:
        out["dw"] = dw
    return out
