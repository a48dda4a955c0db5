"""GPU parity of the token log probabilities (bf16 and 8-bit operands) and of the block quantisation against float64 definitions.

Tolerances, with u = 2^-24.  A logit is a sum of exact products that the tensor core adds up 16 (bf16) or 32 (8 bits) at a time; each
step may cut off up to 2^-23 of what is summed so far: e_x = (d / 16 + 16) 2^-23 sum|h w|, largest over the vocabulary.  On inputs whose
sums are exact in 24 bits (whole numbers times a power of two, "grid") e_x = 0 and the alternatives' ids are the definition's.
2^t is off by 2^-22 relative, t = (x - m) / temperature log2(e) by 2 u |t|, so sum p |t| errors, the running sums and their joins stay below
2^-20 (4 + entropy), and
    lse, logp   e_x / temperature (twice for logp) + 2^-20 (4 + entropy) + 2 u |lse|, + 4 u |logp|
    entropy     e_x / temperature 2 (1 + entropy) + 2^-20 (4 + entropy) (1 + entropy): d entropy / d x_v = -p_v (log p_v + entropy), and the
                sum over v of |p_v (log p_v + entropy)| <= 2 entropy
Gradients: the residual is held as bf16 (its target entry exactly), 2^-9 of each entry at random, and dH is rounded to bf16 (2^-9):
1e-2 in the Frobenius norm, as for the head's loss."""
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
IGN = -100
F8 = torch.float8_e4m3fn


def grid_inputs(T, d, V, seed, spread=2.0):
    """Hidden states and weights on a grid on which every sum of products is exact in 24 bits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randint(-12, 13, (T, d), generator=gen, device="cuda").float()
    w = torch.randint(-12, 13, (V, d), generator=gen, device="cuda").float()
    unit = 2.0 ** round(float(torch.log2(torch.tensor(spread / (49.0 * d ** 0.5)))))
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    tokens[torch.rand(T, generator=gen, device="cuda") < 0.1] = IGN
    return h, w, unit, tokens


def bf16_grid(T, d, V, seed):
    h, w, unit, tokens = grid_inputs(T, d, V, seed)
    return h.to(torch.bfloat16), (w * unit).to(torch.bfloat16), tokens


def fp8_grid(T, d, V, seed):
    h, w, unit, tokens = grid_inputs(T, d, V, seed, spread=1.0)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    pow2 = lambda *s: 2.0 ** torch.randint(-1, 2, s, generator=gen, device="cuda").float()  # noqa: E731
    hs, ws = pow2(T, vp.fp8_blocks(d)), unit * pow2(vp.fp8_blocks(V), vp.fp8_blocks(d))
    full_h = h.double() * orc.spread_columns(hs, d)
    full_w = w.double() * orc.spread_blocks(ws, V, d)
    return (h.to(F8), hs, w.to(F8), ws), (full_h, full_w), tokens


def outputs(T, top):
    f = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    return f(T), f(T), f(T), f(T, top) if top else None, torch.full((T, top), -7, dtype=torch.int32, device="cuda") if top else None


def run(H, W, tokens, top, temperature=1.0):
    T, d = H.shape
    outs = outputs(T, top)
    ws = torch.full((vp.vp_token_logp_workspace_bytes(T, d, W.shape[0], top),), 255, dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_forward(H, W, tokens, temperature, IGN, *outs, ws)
    assert vp.vp_ce_device_status(ws) == 0
    return outs


def run8(ops, tokens, top, temperature=1.0):
    T, d = ops[0].shape
    outs = outputs(T, top)
    ws = torch.full((vp.vp_token_logp_fp8_workspace_bytes(T, d, ops[2].shape[0], top),), 255, dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_fp8_forward(*ops, tokens, temperature, IGN, *outs, ws)
    assert vp.vp_ce_device_status(ws) == 0
    return outs


def within(got, ref, err, what):
    got = got.double()
    over = (got - ref).abs() - err
    assert torch.isfinite(got).all(), what
    assert float(over.max()) <= 0, f"{what}: off by {float((got - ref).abs().flatten()[int(over.argmax())]):.3e}, allowed {float(err.flatten()[int(over.argmax())]):.3e}"


def check(outs, h, w, tokens, top, temperature, e_x):
    """e_x: error of the logits (0: exact, and ids must be the definition's), per token [T]."""
    logp, lse, entropy, top_logp, top_ids = outs
    ref = orc.token_logp(h, w, tokens, temperature, IGN)
    ent = ref["entropy"]
    stat = 2.0 ** -20 * (4 + ent)
    e = e_x / temperature
    e_lse = e + stat + 2 * U * ref["lse"].abs()
    within(lse, ref["lse"], e_lse, "lse")
    within(logp, ref["logp"], 2 * e + stat + 4 * U * ref["logp"].abs(), "logp")
    within(entropy, ent, e * 2 * (1 + ent) + stat * (1 + ent), "entropy")
    assert (logp[~ref["valid"]] == 0).all()
    if not top:
        return
    vals, ids = torch.sort(ref["x"], dim=1, descending=True, stable=True)
    ref_top = ref["logq"].gather(1, ids[:, :top])
    within(top_logp, ref_top, (2 * e + stat)[:, None] + 4 * U * ref_top.abs(), "top_logp")
    got = top_ids.long()
    assert ((got >= 0) & (got < w.shape[0])).all()
    if float(e_x.max()) == 0:
        assert torch.equal(got, ids[:, :top]), "ids"
    else:
        assert all(len(set(r)) == top for r in got.tolist())
        # the chosen column's logit is the rank's own, up to the error of both
        assert ((ref["x"].gather(1, got) - vals[:, :top]).abs() <= 2 * e_x[:, None]).all()


CASES = [  # T, d, V, top, temperature
    (1, 8, 1, 1, 1.0), (1, 64, 5, 5, 1.0), (2, 72, 31, 3, 0.5), (3, 256, 33, 20, 1.0), (1, 2880, 40001, 8, 1.0), (15, 512, 4099, 20, 1.3),
    (16, 64, 127, 1, 1.0), (17, 200, 128, 8, 0.7), (32, 1024, 129, 20, 1.0), (33, 256, 4736, 4, 1.0), (63, 136, 5000, 0, 1.0), (64, 768, 19000, 20, 2.0),
    (65, 64, 1, 1, 1.0), (65, 8, 255, 20, 1.0), (66, 256, 256, 8, 1.0), (128, 512, 257, 20, 0.6), (255, 72, 4099, 5, 1.0), (256, 256, 1000, 0, 1.0),
    (4096, 64, 132000, 0, 1.0), (4100, 64, 70000, 3, 1.0),
    (257, 256, 40000, 20, 1.0), (500, 2880, 9000, 8, 1.0), (1000, 128, 20000, 20, 1.0), (4097, 64, 3000, 8, 1.0), (4500, 192, 17000, 20, 1.0),
]


@pytest.mark.parametrize("T,d,V,top,temperature", CASES)
def test_exact_sums(T, d, V, top, temperature):
    H, W, tokens = bf16_grid(T, d, V, seed=T + d + V)
    check(run(H, W, tokens, top, temperature), H, W, tokens, top, temperature, torch.zeros(T, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("T,d,V,top,temperature", [c for c in CASES if c[1] % 16 == 0])
def test_exact_sums_fp8(T, d, V, top, temperature):
    ops, full, tokens = fp8_grid(T, d, V, seed=T + d + V)
    check(run8(ops, tokens, top, temperature), *full, tokens, top, temperature, torch.zeros(T, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("T,d,V,top", [(1, 2880, 20000, 8), (40, 2048, 10001, 20), (300, 2880, 10001, 20), (700, 7168, 3001, 4)])
def test_ordinary_values(T, d, V, top):
    gen = torch.Generator(device="cuda").manual_seed(T)
    H = torch.randn(T, d, generator=gen, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, d, generator=gen, device="cuda") * (3 / d ** 0.5)).to(torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    e_x = (d / 16 + 16) * 2.0 ** -23 * (H.double().abs() @ W.double().abs().mT).amax(1)
    check(run(H, W, tokens, top, 0.8), H, W, tokens, top, 0.8, e_x)
    # 8 bits, from the operators that make them
    with torch.no_grad():
        hq, hs = vp.rms_norm_fp8(H, torch.ones(d, device="cuda"))
        wq, ws = vp.quantize_blocks_fp8(W)
    full_h, full_w = hq.double() * orc.spread_columns(hs, d), wq.double() * orc.spread_blocks(ws, V, d)
    # the scales' product and the addition to the running sum are fp32, too: three roundings a block
    e_x = (d / 32 + 16 + 3 * d / 128) * 2.0 ** -23 * (full_h.abs() @ full_w.abs().mT).amax(1)
    check(run8((hq, hs, wq, ws), tokens, top, 0.8), full_h, full_w, tokens, top, 0.8, e_x)


def test_peaked_rows_and_large_logits():
    T, d, V = 200, 128, 3000
    h, w, _, tokens = grid_inputs(T, d, V, seed=3)
    H, W = h.to(torch.bfloat16), w.to(torch.bfloat16)                       # logits of several thousand
    for temperature in (1.0, 100.0):
        zero = torch.zeros(T, dtype=torch.float64, device="cuda")
        logp, lse, entropy, top_logp, top_ids = run(H, W, tokens, 20, temperature)
        ref = orc.token_logp(H, W, tokens, temperature, IGN)
        # t = (x - m) / temperature log2(e) reaches thousands: its relative error counts only where 2^t does, |t| < 30
        within(lse, ref["lse"], zero + 2.0 ** -19 + 4 * U * ref["lse"].abs(), "lse")
        within(logp, ref["logp"], zero + 2.0 ** -19 + 8 * U * ref["logp"].abs(), "logp")
        within(entropy, ref["entropy"], 2.0 ** -18 * (1 + ref["entropy"]), "entropy")
        ids = torch.sort(ref["x"], dim=1, descending=True, stable=True)[1][:, :20]
        assert torch.equal(top_ids.long(), ids)


@pytest.mark.parametrize("T", [5, 100])
def test_ties_go_to_the_lowest_id(T):
    V, d = 5000, 64
    H = torch.ones(T, d, device="cuda", dtype=torch.bfloat16)
    W = torch.ones(V, d, device="cuda", dtype=torch.bfloat16)               # every logit is the same
    tokens = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    logp, lse, entropy, top_logp, top_ids = run(H, W, tokens, 20)
    assert torch.equal(top_ids, torch.arange(20, device="cuda", dtype=torch.int32).expand(T, 20))
    want = torch.log(torch.tensor(float(V), dtype=torch.float64))
    assert float((entropy.double().cpu() - want).abs().max()) < 1e-5 and float((logp.double().cpu() + want).abs().max()) < 1e-5
    # the best columns at the end, in falling order of id: every slice improves the list
    W[-40:] *= 2
    _, _, _, _, top_ids = run(H, W, tokens, 20)
    assert torch.equal(top_ids, torch.arange(V - 40, V - 20, device="cuda", dtype=torch.int32).expand(T, 20))


@pytest.mark.parametrize("T", [5, 100, 600])
def test_zero_rows(T):
    """Hidden states of padding: every logit is a zero, some of them negative ones."""
    V, d = 40000, 64
    H = torch.zeros(T, d, device="cuda", dtype=torch.bfloat16)
    H[1::2] = -0.0
    W = torch.randn(V, d, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").to(torch.bfloat16)
    _, _, entropy, top_logp, top_ids = run(H, W, torch.zeros(T, dtype=torch.int32, device="cuda"), 20)
    assert torch.equal(top_ids, torch.arange(20, device="cuda", dtype=torch.int32).expand(T, 20))
    assert float((entropy.double() - torch.log(torch.tensor(float(V), dtype=torch.float64))).abs().max()) < 1e-5
    assert float((top_logp + entropy[:, None]).abs().max()) < 1e-5


@pytest.mark.parametrize("T", [7, 300])
def test_rising_logits(T):
    """The worst order for the lists: every column is better than all before it."""
    V, d = 20000, 64
    W = torch.zeros(V, d, device="cuda")
    W[:, 0], W[:, 1] = torch.arange(V, device="cuda") // 128, torch.arange(V, device="cuda") % 128
    H = torch.zeros(T, d, device="cuda")
    H[:, 0], H[:, 1] = 1, 1 / 128
    tokens = torch.zeros(T, dtype=torch.int32, device="cuda")
    _, _, _, _, top_ids = run(H.to(torch.bfloat16), W.to(torch.bfloat16), tokens, 20)
    assert torch.equal(top_ids, torch.arange(V - 1, V - 21, -1, device="cuda", dtype=torch.int32).expand(T, 20))


@pytest.mark.parametrize("T", [6, 90])
def test_nan_stays_in_its_row_or_column(T):
    H, W, tokens = bf16_grid(T, 64, 3000, seed=T)
    tokens.fill_(17)
    clean = run(H, W, tokens, 8)
    H[2, 5] = float("nan")
    logp, lse, entropy, top_logp, top_ids = run(H, W, tokens, 8)
    for a in (logp, lse, entropy):
        assert torch.isnan(a[2]) and torch.isfinite(a[:2]).all() and torch.isfinite(a[3:]).all()
    assert (top_ids[2] == -1).all() and (top_logp[2] == -float("inf")).all()
    rest = [i for i in range(T) if i != 2]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip((logp, lse, entropy, top_logp, top_ids), clean))
    H[2, 5] = 0
    W[40:80] = float("nan")                                                 # whole slices of a thread, and parts
    logp, lse, entropy, _, top_ids = run(H, W, tokens, 8)
    assert torch.isnan(lse).all() and torch.isnan(entropy).all() and torch.isnan(logp).all()
    assert ((top_ids < 40) | (top_ids >= 80)).all() and (top_ids >= 0).all()


@pytest.mark.parametrize("T", [6, 90])
def test_tokens_outside_and_left_out(T):
    H, W, tokens = bf16_grid(T, 64, 300, seed=T)
    tokens[0], tokens[1] = 300, -5
    outs = outputs(T, 3)
    ws = torch.empty(vp.vp_token_logp_workspace_bytes(T, 64, 300, 3), dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, *outs, ws)
    assert vp.vp_ce_device_status(ws) == 1 and (outs[0][:2] == 0).all()
    # no tokens: the same entropy, lse and alternatives
    only = outputs(T, 3)
    vp.vp_token_logp_forward(H, W, None, 1.0, IGN, None, *only[1:], ws)
    assert vp.vp_ce_device_status(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(outs[1:], only[1:]))
    # and what is not asked for is not written
    lone = outputs(T, 0)
    ws = torch.empty(vp.vp_token_logp_workspace_bytes(T, 64, 300, 0), dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, lone[0], None, None, None, None, ws)
    assert torch.equal(lone[0], outs[0]) and torch.isnan(lone[1]).all()


def test_nothing_behind_the_last_token_or_workspace():
    for T in (3, 70):
        H, W, tokens = bf16_grid(T, 64, 5000, seed=T)
        n = vp.vp_token_logp_workspace_bytes(T, 64, 5000, 4)
        ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
        big = [torch.full((T + 50,), 5.0, device="cuda") for _ in range(3)]
        tl, ti = torch.full((T + 50, 4), 5.0, device="cuda"), torch.full((T + 50, 4), 5, dtype=torch.int32, device="cuda")
        vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, *[b[:T] for b in big], tl[:T], ti[:T], ws[:n])
        assert (ws[n:] == 77).all() and all((b[T:] == 5).all() for b in big) and (tl[T:] == 5).all() and (ti[T:] == 5).all()


@pytest.mark.parametrize("T", [9, 1000])
def test_repeats_streams_and_graphs(T):
    H, W, tokens = bf16_grid(T, 256, 9000, seed=T)
    first = run(H, W, tokens, 8, 0.9)
    second = run(H, W, tokens, 8, 0.9)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    ws = torch.empty(vp.vp_token_logp_workspace_bytes(T, 256, 9000, 8), dtype=torch.uint8, device="cuda")
    outs = outputs(T, 8)
    graph = torch.cuda.CUDAGraph()
    vp.vp_token_logp_forward(H, W, tokens, 0.9, IGN, *outs, ws)
    with torch.cuda.graph(graph):
        vp.vp_token_logp_forward(H, W, tokens, 0.9, IGN, *outs, ws)
    for _ in range(2):
        for o in outs:
            o.fill_(0)
        ws.fill_(255)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = outputs(T, 8)
    ws2 = torch.empty_like(ws)
    with torch.cuda.stream(s):
        vp.vp_token_logp_forward(H, W, tokens, 0.9, IGN, *other, ws2)
    vp.vp_token_logp_forward(H, W, tokens, 0.9, IGN, *outs, ws)             # both at once
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, outs, other))


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("T,d,V,temperature", [(1, 64, 300, 1.0), (5, 256, 1000, 0.7), (130, 72, 600, 1.0), (300, 512, 3001, 1.4), (700, 320, 9000, 1.0)])
def test_gradients(T, d, V, temperature):
    gen = torch.Generator(device="cuda").manual_seed(T)
    H = torch.randn(T, d, generator=gen, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, d, generator=gen, device="cuda") * (2 / d ** 0.5)).to(torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    if T > 10:
        tokens[3], tokens[4] = IGN, V + 5
        tokens[5:9] = tokens[9]                                             # the same target several times
    dlogp, dent = torch.randn(T, generator=gen, device="cuda"), torch.randn(T, generator=gen, device="cuda")
    _, lse, entropy, _, _ = (outs := outputs(T, 0))
    ws = torch.empty(vp.vp_token_logp_workspace_bytes(T, d, V, 0), dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_forward(H, W, tokens, temperature, IGN, *outs, ws)
    chunk, block_v = 256, 512
    ws = torch.empty(vp.vp_ce_workspace_bytes(chunk, d, block_v), dtype=torch.uint8, device="cuda")
    for u, v in ((dlogp, None), (None, dent), (dlogp, dent)):
        dH, dW = torch.full_like(H, float("nan")), torch.full((V, d), float("nan"), device="cuda")
        vp.vp_token_logp_backward(H, W, tokens, lse, entropy if v is not None else None, u, v, temperature, IGN, dH, dW, block_v, chunk, False, ws)
        rH, rW, _ = orc.token_logp_grad(H, W, tokens, u, v, temperature, IGN)
        assert rel(dH, rH) <= 1e-2 and rel(dW, rW) <= 1e-2
        # accumulated into what is there, and each gradient by itself
        more = dW.clone()
        vp.vp_token_logp_backward(H, W, tokens, lse, entropy, u, v, temperature, IGN, None, more, block_v, chunk, True, ws)
        assert rel(more, 2 * rW) <= 1e-2
        alone = torch.empty_like(dH)
        vp.vp_token_logp_backward(H, W, tokens, lse, entropy, u, v, temperature, IGN, alone, None, block_v, chunk, False, ws)
        assert torch.equal(alone, dH)


def test_log_probability_gradient_is_the_loss_gradient():
    """Without entropy and temperature the operator is the head's loss with its sign turned."""
    H, W, tokens = bf16_grid(300, 256, 2000, seed=1)
    a, b = H.clone().requires_grad_(), W.clone().requires_grad_()
    c, e = H.clone().requires_grad_(), W.clone().requires_grad_()
    up = torch.randn(300, device="cuda")
    (vp.token_log_probs(a, b, tokens, block_v=512).logp * up).sum().backward()
    (-vp.vocab_proj_cross_entropy(c, e, tokens, block_v=512) * up).sum().backward()
    assert rel(a.grad, c.grad.double()) < 1e-3 and rel(b.grad, e.grad.double()) < 1e-3


def test_autograd():
    H, W, tokens = bf16_grid(130, 64, 700, seed=2)
    H.requires_grad_(), W.requires_grad_()
    out = vp.token_log_probs(H, W, tokens.long(), top_k=3, temperature=0.8, block_v=256)
    assert not out.top_logp.requires_grad and out.logp.requires_grad and out.entropy.requires_grad
    up = torch.randn(130, device="cuda")
    ((out.logp * up).sum() + 0.3 * out.entropy.sum()).backward()
    rH, rW, _ = orc.token_logp_grad(H.detach(), W.detach(), tokens, up, torch.full((130,), 0.3, device="cuda"), 0.8)
    assert rel(H.grad, rH) <= 1e-2 and rel(W.grad, rW) <= 1e-2
    # entropy alone, without tokens; the accumulation buffer; a frozen weight
    H.grad = W.grad = None
    acc = torch.zeros(700, 64, device="cuda")
    vp.token_log_probs(H, W, block_v=256, dW_accum=acc).entropy.sum().backward()
    rH, rW, _ = orc.token_logp_grad(H.detach(), W.detach(), None, None, torch.ones(130, device="cuda"), 1.0)
    assert W.grad is None and rel(acc, rW) <= 1e-2 and rel(H.grad, rH) <= 1e-2
    H.grad = None
    vp.token_log_probs(H, W.detach(), tokens, block_v=256).logp.sum().backward()
    assert H.grad is not None
    (g,) = torch.autograd.grad(vp.token_log_probs(H, W, tokens, block_v=256).logp.square().sum(), H, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()


def test_captured_gradients():
    """Forward and backward in one graph, replayed on new inputs.  (No eager graph of the same leaves may live meanwhile: torch keeps
    their accumulation on the stream of that one, outside the capture.)"""
    H, W, tokens = bf16_grid(130, 64, 700, seed=4)
    H.requires_grad_(), W.requires_grad_()
    x, r = torch.randn(130, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True), torch.randn(130, 64, device="cuda", dtype=torch.bfloat16)

    def step():
        y, z = vp.rms_norm(x, None, r)
        out = vp.token_log_probs(H + y, W, tokens, top_k=2, block_v=256)
        return torch.autograd.grad(out.logp.sum() + 0.1 * out.entropy.sum() + z.sum(), (H, W, x))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    with torch.no_grad():
        H.neg_(), r.mul_(2)
    graph.replay()
    got = [g.clone() for g in captured]
    assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_empty():
    H, W = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(10, 64, device="cuda", dtype=torch.bfloat16)
    W.requires_grad_()
    out = vp.token_log_probs(H, W, torch.empty(0, dtype=torch.int32, device="cuda"), top_k=2, block_v=256)
    assert out.logp.shape == (0,) and out.top_ids.shape == (0, 2)
    out.logp.sum().backward()
    assert (W.grad == 0).all()


@pytest.mark.parametrize("T", [4, 100])
@pytest.mark.parametrize("fp8", [False, True])
def test_a_lost_copy_ends_in_the_status_word(T, fp8):
    ops, _, tokens = fp8_grid(T, 1024, 3000, seed=1)
    H, W, _ = bf16_grid(T, 1024, 3000, seed=1)
    args = ops if fp8 else (H, W)
    call = vp.vp_token_logp_fp8_forward if fp8 else vp.vp_token_logp_forward
    size = vp.vp_token_logp_fp8_workspace_bytes if fp8 else vp.vp_token_logp_workspace_bytes
    ws = torch.empty(size(T, 1024, 3000, 4), dtype=torch.uint8, device="cuda")
    want = outputs(T, 4)
    call(*args, tokens, 1.0, IGN, *want, ws)
    before = vp.vp_ce_set_wait_limit_ns(20_000_000)
    try:
        vp.vp_token_logp_debug_drop(2)
        call(*args, tokens, 1.0, IGN, *outputs(T, 4), ws)
        assert vp.vp_ce_device_status(ws) & 2
    finally:
        vp.vp_ce_set_wait_limit_ns(before)
        vp.vp_token_logp_debug_drop(-1)
    again = outputs(T, 4)
    call(*args, tokens, 1.0, IGN, *again, ws)                               # the next call starts clean
    assert vp.vp_ce_device_status(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_refusals():
    H, W, tokens = bf16_grid(4, 64, 300, seed=1)
    outs = outputs(4, 2)
    ws = torch.empty(vp.vp_token_logp_workspace_bytes(4, 64, 300, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError):
        vp.vp_token_logp_forward(H.half(), W, tokens, 1.0, IGN, *outs, ws)
    with pytest.raises(TypeError):
        vp.vp_token_logp_forward(H, W, tokens.long(), 1.0, IGN, *outs, ws)
    with pytest.raises(ValueError):
        vp.vp_token_logp_forward(H, W, None, 1.0, IGN, *outs, ws)
    with pytest.raises(ValueError):
        vp.vp_token_logp_forward(H, W[:, :56], tokens, 1.0, IGN, *outs, ws)
    for bad in (0.0, -1.0, float("nan"), 1e-7, 1e7):
        with pytest.raises(vp.VpceError):
            vp.vp_token_logp_forward(H, W, tokens, bad, IGN, *outs, ws)
    with pytest.raises(vp.VpceError):
        vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, *outs, ws[:64])
    with pytest.raises(ValueError):
        vp.token_log_probs(H, W, tokens, top_k=21)
    with pytest.raises(ValueError):
        vp.token_log_probs(H, W[:5], tokens, top_k=6)
    with pytest.raises(ValueError):
        vp.token_log_probs(H[:, :60].contiguous(), W[:, :60].contiguous(), tokens)
    with pytest.raises(TypeError):
        vp.token_log_probs(H.float(), W.float(), tokens)
    ops, _, _ = fp8_grid(4, 64, 300, seed=1)
    with pytest.raises(ValueError):
        vp.token_log_probs_fp8(ops[0], ops[1][:, :0], ops[2], ops[3], tokens)
    with pytest.raises(TypeError):
        vp.token_log_probs_fp8(ops[0].float(), *ops[1:], tokens)
    ws2 = torch.empty(vp.vp_ce_workspace_bytes(128, 64, 256), dtype=torch.uint8, device="cuda")
    dH = torch.empty_like(H)
    with pytest.raises(vp.VpceError):                                       # no upstream gradient
        vp.vp_token_logp_backward(H, W, tokens, outs[1], outs[2], None, None, 1.0, IGN, dH, None, 256, 128, False, ws2)
    with pytest.raises(vp.VpceError):                                       # an entropy gradient without the entropy
        vp.vp_token_logp_backward(H, W, tokens, outs[1], None, None, outs[0], 1.0, IGN, dH, None, 256, 128, False, ws2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (128, 128, 0), (129, 257, 0), (300, 1000, 24), (500, 2880, 0), (77, 1111, 3), (1000, 64, 64)])
def test_quantize_blocks(rows, d, pad, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randn(rows, d + pad, generator=gen, device="cuda").mul_(0.02).to(dtype)[:, :d]
    if rows > 1:
        w[0, 0] = float("nan")
    if rows > 256:
        w[128:256] = 0
    q = torch.zeros(rows, d + pad, device="cuda").to(F8)[:, :d]
    s = torch.full((vp.fp8_blocks(rows), vp.fp8_blocks(d)), float("nan"), device="cuda")
    vp.vp_fp8_quantize_blocks(w, q, s)
    clean = torch.nan_to_num(w.double())                                    # the NaN takes no part in the maximum
    ref = orc.block_scales(clean)
    assert ((s.double() - ref).abs() <= ref * 4 * U).all()
    spread = orc.spread_blocks(s, rows, d)
    back = q.double() * spread
    if rows > 1:
        assert torch.isnan(back[0, 0])
        back[0, 0] = 0
    err = torch.maximum(clean.abs() * 2.0 ** -4 * 1.0001, spread * 2.0 ** -10)
    assert ((back - clean).abs() <= err).all()
    if rows > 256:
        assert (s[1] == 1).all() and (back[128:256] == 0).all()


def test_quantize_more_rows_than_one_launch_takes():
    rows = 65535 * 128 + 130
    w = torch.ones(rows, 1, device="cuda", dtype=torch.bfloat16)
    w[-130:] = 3
    q, s = vp.quantize_blocks_fp8(w)
    assert (q.float() == 448).all() and (s[:-2] == torch.tensor(1.0) / 448).all()
    assert ((s[-2:] - 3 / 448).abs() <= 3 / 448 * 4 * U).all()


def test_quantize_blocks_refusals():
    w = torch.zeros(4, 64, device="cuda")
    q, s = torch.zeros(4, 64, device="cuda").to(F8), torch.zeros(1, 1, device="cuda")
    with pytest.raises(TypeError):
        vp.vp_fp8_quantize_blocks(w.double(), q, s)
    with pytest.raises(TypeError):
        vp.vp_fp8_quantize_blocks(w, w, s)
    with pytest.raises(ValueError):
        vp.vp_fp8_quantize_blocks(w, q, torch.zeros(2, device="cuda"))
    q2, s2 = vp.quantize_blocks_fp8(torch.nn.Parameter(w.t()))
    assert q2.shape == (64, 4) and s2.shape == (1, 1) and (s2 == 1).all()


def test_forward_without_backward_frees_its_memory():
    """A graph that is dropped without a backward pass holds nothing afterwards."""
    H, W = (torch.randn(n, 256, device="cuda", dtype=torch.bfloat16, requires_grad=True) for n in (96, 1000))
    tokens = torch.arange(96, device="cuda")

    def step():
        vp.token_log_probs(H, W, tokens, top_k=4)

    step()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for _ in range(4):
        step()
    assert torch.cuda.memory_allocated() == before


@pytest.mark.parametrize("T,V,T_chunk", [(40, 20011, None), (0, 500, None), (300, 70001, 128)])
def test_default_strips(T, V, T_chunk):
    """Gradients without a given strip width: one strip wider than 8192 columns, no tokens, several chunks."""
    H, W, tokens = bf16_grid(T, 64, V, seed=3)
    H.requires_grad_(), W.requires_grad_()
    out = vp.token_log_probs(H, W, tokens, temperature=0.8, T_chunk=T_chunk)
    up = torch.randn(T, device="cuda")
    ((out.logp * up).sum() + 0.3 * out.entropy.sum()).backward()
    if T == 0:
        assert H.grad.shape == (0, 64) and not W.grad.any()
        return
    rH, rW, _ = orc.token_logp_grad(H.detach(), W.detach(), tokens, up, torch.full((T,), 0.3, device="cuda"), 0.8)
    assert rel(H.grad, rH) <= 1e-2 and rel(W.grad, rW) <= 1e-2
