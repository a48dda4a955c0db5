"""Token log probabilities where a wait runs out on workspaces that hold anything, beside NaN, at the ends of the temperatures, with strips
as wide as the default takes them, and calls that are refused."""
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc
from test_gpu_token_logp import F8, IGN, bf16_grid, check, fp8_grid, outputs, run, run8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,V,top", [(4, 1024, 3000, 4), (40, 1024, 3000, 0), (100, 1024, 3000, 20), (300, 1024, 3000, 0), (5000, 512, 20000, 20)])
def test_a_lost_copy_on_a_workspace_of_arbitrary_bytes(T, d, V, top, fp8):
    """Nothing that the workspace held is taken for a state or a count of candidates: no results, and the next call starts clean.
    (5000 tokens: two chunks of two strips or more.)"""
    ops, _, tokens = fp8_grid(T, d, V, seed=1)
    H, W, _ = bf16_grid(T, d, V, seed=1)
    args = ops if fp8 else (H, W)
    call = vp.vp_token_logp_fp8_forward if fp8 else vp.vp_token_logp_forward
    n = (vp.vp_token_logp_fp8_workspace_bytes if fp8 else vp.vp_token_logp_workspace_bytes)(T, d, V, top)

    def workspace():                                        # as counts: 1061109567
        ws = torch.full((n + 4096,), 0x3f, dtype=torch.uint8, device="cuda")
        return ws, ws[:n]

    want = outputs(T, top)
    call(*args, tokens, 1.0, IGN, *want, workspace()[1])
    before = vp.vp_ce_set_wait_limit_ns(20_000_000)
    try:
        whole, ws = workspace()
        got = outputs(T, top)
        vp.vp_token_logp_debug_drop(2)
        call(*args, tokens, 1.0, IGN, *got, ws)
        assert vp.vp_ce_device_status(ws) & 2
    finally:
        vp.vp_ce_set_wait_limit_ns(before)
        vp.vp_token_logp_debug_drop(-1)
    logp, lse, entropy, top_logp, top_ids = got
    assert torch.isnan(lse).all() and torch.isnan(entropy).all()
    assert torch.isnan(logp[tokens != IGN]).all() and (logp[tokens == IGN] == 0).all()
    if top:
        assert (top_ids == -1).all() and (top_logp == -float("inf")).all()
    assert (whole[n:] == 0x3f).all()
    again = outputs(T, top)
    call(*args, tokens, 1.0, IGN, *again, ws)
    assert vp.vp_ce_device_status(ws) == 0
    assert all(a is None or torch.equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,V,top", [(7, 128, 5), (65, 128, 5), (300, 128, 20), (200, 256, 5), (1000, 1000, 8)])
def test_alternatives_beside_columns_of_nan(T, V, top, fp8):
    """A NaN is not an alternative and takes no other column's place: four neighbours of NaN (all that one bound looks at) at every
    place, and single ones.  Ids are the definition's, the sums being exact."""
    (hq, hs, wq, ws), (full_h, full_w), tokens = fp8_grid(T, 128, V, seed=T + V)
    H, W, _ = bf16_grid(T, 128, V, seed=T + V)
    x = full_h @ full_w.mT if fp8 else H.double() @ W.double().mT
    for first in (0, 28, 64, 124):
        gone = torch.zeros(V, dtype=torch.bool, device="cuda")
        gone[first:first + 4] = True
        gone[::17] = True
        if fp8:
            bad = wq.view(torch.uint8).clone()
            bad[gone, 3] = 0x7f
            _, lse, _, top_logp, top_ids = run8((hq, hs, bad.view(F8), ws), tokens, top)
        else:
            bad = W.clone()
            bad[gone, 3] = float("nan")
            _, lse, _, top_logp, top_ids = run(H, bad, tokens, top)
        want = torch.sort(x.masked_fill(gone, -float("inf")), dim=1, descending=True, stable=True)[1][:, :top]
        assert torch.equal(top_ids.long(), want)
        assert torch.isnan(lse).all() and torch.isnan(top_logp).all()


@pytest.mark.parametrize("T", [70, 130])
@pytest.mark.parametrize("temperature,unit,size", [(0.01, 2.0 ** -10, 32), (0.01, 2.0 ** -10, 512), (2.0 ** -6, 2.0 ** -10, 32), (2.0 ** -6, 2.0 ** -10, 512),
                                                   (0.1, 2.0 ** -7, 512), (1.0, 2.0 ** -4, 32), (64.0, 2.0 ** -4, 32), (100.0, 2.0 ** -4, 32)])
def test_gradients_at_the_ends_of_the_temperatures(T, temperature, unit, size):
    """Logits of 32 or 512 and a spread that leaves many columns likely at each temperature, on sums that are exact; lse and entropy from the
    definition, rounded once.

    With s = x / temperature - lse the residual is (dlogp (onehot - p) - dent p (s + entropy)) / temperature, p = exp(s).  lse, its product
    with log2(e), 1 / temperature and its product with log2(e) are rounded apart, then s: s is off by 2^-24 (2 |lse| + 2 |x / temperature| +
    2 |s|), p by as much and 2^-22 relative (the hardware's exponential).  s + entropy comes from lse, entropy, their difference and
    its product with dent, and logits times a twice rounded factor: 2^-24 (3 (|lse| + entropy) + 2 |x / temperature| + its own size);
    the products 2^-21.  So every entry
    lies between two numbers, and what bf16 makes of it between what it makes of those (the target's entry is held exactly).  To that
    the tensor core's cuts (2^-23 a step of 16 columns or tokens) and the result's bf16 (2^-8) are added."""
    d, V = 64, 2000
    gen = torch.Generator(device="cuda").manual_seed(T)
    H = torch.randint(-12, 13, (T, d), generator=gen, device="cuda").float() / 8
    W = torch.randint(-12, 13, (V, d), generator=gen, device="cuda").float() * unit
    H[:, 0], W[:, 0] = size, 1
    H, W = H.to(torch.bfloat16), W.to(torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    tokens[3] = IGN
    u, v = torch.randn(T, generator=gen, device="cuda"), torch.randn(T, generator=gen, device="cuda")
    ref = orc.token_logp(H, W, tokens, temperature, IGN)
    lse, entropy = ref["lse"].float(), ref["entropy"].float()
    s = ref["logq"]
    p = torch.exp(s)
    c = s + ref["entropy"][:, None]
    e_s = 2.0 ** -24 * (2 * ref["lse"].abs()[:, None] + 2 * (ref["x"] / temperature).abs() + 2 * s.abs())
    e_p = e_s + 2.0 ** -22
    e_c = 2.0 ** -24 * (3 * (ref["lse"].abs() + ref["entropy"])[:, None] + 2 * (ref["x"] / temperature).abs() + c.abs())
    ws = torch.empty(vp.vp_ce_workspace_bytes(256, d, 512), dtype=torch.uint8, device="cuda")
    h, w = H.double().abs(), W.double().abs()
    for a, b in ((u, None), (None, v), (u, v)):
        dH, dW = torch.empty_like(H), torch.empty(V, d, device="cuda")
        vp.vp_token_logp_backward(H, W, tokens, lse, entropy if b is not None else None, a, b, temperature, IGN, dH, dW, 512, 256, False, ws)
        rH, rW, G = orc.token_logp_grad(H, W, tokens, a, b, temperature, IGN)
        first = torch.zeros(T, dtype=torch.float64, device="cuda") if a is None else torch.where(ref["valid"], a.double().abs(), 0.0)
        second = torch.zeros_like(first) if b is None else b.double().abs()
        e_g = p * (e_p * (first[:, None] + second[:, None] * c.abs()) + second[:, None] * e_c) / temperature + 2.0 ** -21 * G.abs()
        at = torch.zeros_like(G, dtype=torch.bool)
        at[ref["valid"]] = at[ref["valid"]].scatter(1, tokens.long()[ref["valid"]][:, None], True)
        low, high = (torch.where(at, g, g.to(torch.bfloat16).double()) for g in (G - e_g, G + e_g))
        mid, half = (low + high) / 2, (high - low) / 2
        steps = (512 / 16 + 8) * 2.0 ** -23
        for got, want, free, total in ((dH, mid @ W.double(), half @ w, G.abs() @ w), (dW, mid.mT @ H.double(), half.mT @ h, G.abs().mT @ h)):
            allowed = free + steps * total + (2.0 ** -8 * (1 + 2.0 ** -8) * want.abs() if got is dH else 0)
            err = (got.double() - want).abs()
            assert (err <= allowed).all(), float((err / allowed).nan_to_num().max())


def test_gradients_outside_the_temperatures_are_refused():
    H, W, tokens = bf16_grid(70, 64, 300, seed=1)
    ws = torch.empty(vp.vp_ce_workspace_bytes(128, 64, 512), dtype=torch.uint8, device="cuda")
    lse, entropy, u = (torch.zeros(70, device="cuda") for _ in range(3))
    for temperature in (1e-6, 0.0099, 100.5, 1e6, float("nan")):
        with pytest.raises(vp.VpceError):
            vp.vp_token_logp_backward(H, W, tokens, lse, entropy, u, u, temperature, IGN, torch.empty_like(H), None, 512, 128, False, ws)
    H.requires_grad_()
    for temperature in (1e-3, 1e3):
        out = vp.token_log_probs(H, W, tokens, temperature=temperature)     # the forward call's range is wider
        assert torch.isfinite(out.logp).all()
        with pytest.raises(ValueError, match="temperature"):
            out.logp.sum().backward()


def test_default_strips_hold_their_sums():
    """dH where a strip's sum is far larger than what is left of it in the end (rows of W with a common mean): p sums to 1 over columns
    near 1, and -1 of the target's comes against it.

    A strip of n columns is n / 16 steps of the tensor core, each of which may cut off 2^-23 of the sum, itself at most A = sum |G W|: at the
    default's most, 16384 columns, 2^-13 A.  Beside that G is rounded to bf16 (half a step, 2^-8 of each entry, evenly spread: six times
    2^-8 / sqrt(3) sqrt(sum G^2 W^2); the target's entry exactly), the strips are added up in fp32 (13 times 2^-24 A), and the result is
    rounded to bf16 (2^-8)."""
    T, d, V = 200, 128, 201088
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = (1 + 0.1 * torch.randn(V, d, generator=gen, device="cuda")).to(torch.bfloat16)
    H = torch.randn(T, d, generator=gen, device="cuda")
    H = (H - H.mean(1, keepdim=True)).to(torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    H.requires_grad_()
    vp.token_log_probs(H, W, tokens).logp.sum().backward()
    dH, _, G = orc.token_logp_grad(H.detach(), W, tokens, torch.ones(T, device="cuda"), None, 1.0)
    A = G.abs() @ W.double().abs()
    G.scatter_(1, tokens.long()[:, None], 0.0)
    Q = (G.square() @ W.double().square()).sqrt()
    err = (H.grad.double() - dH).abs()
    allowed = (2.0 ** -13 + 13 * 2.0 ** -24) * A + 6 * 2.0 ** -8 / 3 ** 0.5 * Q + 2.0 ** -8 * dH.abs() * (1 + 2.0 ** -8)
    assert (err <= allowed).all(), float((err / allowed).max())


def test_scales_and_gradients_of_another_shape_are_refused():
    """As many elements in another order are another matrix."""
    T, d, V = 256, 384, 640                                                 # Hs [256, 3], Ws [5, 3]
    (hq, hs, wq, ws), _, tokens = fp8_grid(T, d, V, seed=1)
    vp.token_log_probs_fp8(hq, hs, wq, ws, tokens)
    for bad in ((hq, hs.t(), wq, ws), (hq, hs, wq, ws.t()), (hq, hs.reshape(-1), wq, ws), (hq, hs, wq, ws.reshape(3, 5))):
        with pytest.raises(ValueError, match="must be"):
            vp.token_log_probs_fp8(*bad, tokens)
    with pytest.raises(ValueError, match="must be"):
        vp.vp_fp8_quantize_blocks(torch.zeros(V, d, device="cuda"), torch.empty_like(wq), ws.t().contiguous())
    with pytest.raises(ValueError, match="must be"):
        vp.vp_rms_forward_fp8(torch.zeros(T, d, device="cuda"), None, None, 1e-6, torch.empty_like(hq), hs.t().contiguous(), None, None)
    H, W, _ = bf16_grid(T, d, V, seed=1)
    outs = outputs(T, 2)
    room = torch.empty(vp.vp_token_logp_workspace_bytes(T, d, V, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="must be"):
        vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, *outs[:4], outs[4].reshape(2, T), room)
    room = torch.empty(vp.vp_ce_workspace_bytes(256, d, 256), dtype=torch.uint8, device="cuda")
    vp.vp_token_logp_forward(H, W, tokens, 1.0, IGN, *outs[:3], None, None, torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    for dH, dW in ((torch.empty(d, T, device="cuda", dtype=torch.bfloat16), None), (None, torch.zeros(d, V, device="cuda"))):
        with pytest.raises(ValueError, match="must be"):
            vp.vp_token_logp_backward(H, W, tokens, outs[1], None, outs[0], None, 1.0, IGN, dH, dW, 256, 256, False, room)
    H.requires_grad_()
    with pytest.raises(ValueError, match="must be"):
        vp.token_log_probs(H, W, tokens, block_v=256, dW_accum=torch.zeros(d, V, device="cuda")).logp.sum().backward()


def test_scales_that_require_a_gradient_are_refused():
    (hq, hs, wq, ws), _, tokens = fp8_grid(4, 128, 300, seed=1)
    for i in (0, 1):
        a, b = (hs.clone().requires_grad_(i == 0), ws.clone().requires_grad_(i == 1))
        with pytest.raises(RuntimeError, match="no gradient"):
            vp.token_log_probs_fp8(hq, a, wq, b, tokens)
        with torch.no_grad():
            assert torch.isfinite(vp.token_log_probs_fp8(hq, a, wq, b, tokens).logp).all()


@pytest.mark.parametrize("T", [8, 100])
def test_tokens_that_32_bits_do_not_hold(T):
    """A 64-bit token outside 32 bits is a token outside the vocabulary, not the one that its low half names."""
    H, W, _ = bf16_grid(T, 64, 300, seed=T)
    tokens = torch.arange(T, device="cuda") % 300
    far = tokens.clone()
    far[0], far[1], far[2], far[3], far[4] = 2 ** 32 + 5, -2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1, 2 ** 63 - 1
    a, b = vp.token_log_probs(H, W, tokens), vp.token_log_probs(H, W, far)
    assert (b.logp[:5] == 0).all() and torch.equal(a.logp[5:], b.logp[5:]) and torch.equal(a.entropy, b.entropy)
    H.requires_grad_()
    vp.token_log_probs(H, W, far).logp.sum().backward()
    assert (H.grad[:5] == 0).all() and (H.grad[5:] != 0).any(1).all()
    ops, _, _ = fp8_grid(T, 64, 300, seed=T)
    assert (vp.token_log_probs_fp8(*ops, far).logp[:5] == 0).all()
    for dtype in (torch.uint8, torch.int8, torch.int16):
        few = (torch.arange(T, device="cuda") % 100).to(dtype)
        assert torch.equal(vp.token_log_probs(H, W, few).logp, vp.token_log_probs(H, W, few.int()).logp)


def test_tokens_and_ignore_index_that_are_none_are_refused():
    H, W, tokens = bf16_grid(4, 64, 300, seed=1)
    ops, _, _ = fp8_grid(4, 64, 300, seed=1)
    for call in (lambda t, **k: vp.token_log_probs(H, W, t, **k), lambda t, **k: vp.token_log_probs_fp8(*ops, t, **k)):
        for bad in (tokens.float(), tokens.bool(), [1, 2, 3, 4]):
            with pytest.raises(TypeError):
                call(bad)
        for bad in (2 ** 31, -2 ** 31 - 1, 2 ** 32 - 100):
            with pytest.raises(ValueError, match="ignore_index"):
                call(tokens, ignore_index=bad)


@pytest.mark.parametrize("temperature", [1e-6, 1e-3, 1e6])
@pytest.mark.parametrize("T", [5, 100])
def test_temperatures_of_the_forward_pass(T, temperature):
    H, W, tokens = bf16_grid(T, 64, 5000, seed=T)
    check(run(H, W, tokens, 8, temperature), H, W, tokens, 8, temperature, torch.zeros(T, dtype=torch.float64, device="cuda"))
    ops, full, tokens = fp8_grid(T, 64, 5000, seed=T)
    check(run8(ops, tokens, 8, temperature), *full, tokens, 8, temperature, torch.zeros(T, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("T", [1, 16, 17, 64, 65])
@pytest.mark.parametrize("d", [16, 16384])
def test_narrowest_and_widest_rows_in_8_bits(T, d):
    ops, full, tokens = fp8_grid(T, d, 700, seed=T)
    check(run8(ops, tokens, 5), *full, tokens, 5, 1.0, torch.zeros(T, dtype=torch.float64, device="cuda"))
