"""The operators from the residual stream to log probabilities where element offsets pass 2^31: the last rows of arrays of more than
2^31 elements against the same rows alone, and a weight of that size against float64 at its last columns.

Tolerances of the log probabilities as in test_gpu_token_logp.py: a logit is off by e_x = (d / 16 + 16) 2^-23 sum|h w| at most (8 bits: d / 32
steps, and three roundings for each block of 128), lse and the chosen logit by as much each; statistics by 2^-20 (4 + entropy).  (The
likely column's logit here is a sum of 8192 terms of one sign, 819: every step cuts off in the same direction.)"""
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
IGN = -100


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def fill(*shape, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("rows,d", [(270000, 8192), (2100000, 1024), (1940000, 1111), (34000000, 64)])
def test_rms_norm(rows, d):
    assert rows * d > 1 << 31
    tail = slice(rows - 700, rows)
    x, r, w = fill(rows, d), fill(rows, d, seed=1), fill(d, seed=2)
    y, z, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    vp.vp_rms_forward(x, r, w, 1e-6, y, z, rstd)
    few = [t[tail].clone() for t in (x, r)]
    y1, z1, rs1 = torch.empty_like(few[0]), torch.empty_like(few[0]), torch.empty(700, device="cuda")
    vp.vp_rms_forward(*few, w, 1e-6, y1, z1, rs1)
    assert torch.equal(z[tail], z1) and torch.equal(rstd[tail], rs1) and torch.equal(y[tail], y1)
    q, s = torch.empty(rows, d, device="cuda", dtype=F8), torch.empty(rows, vp.fp8_blocks(d), device="cuda")
    vp.vp_rms_forward_fp8(x, r, w, 1e-6, q, s, None, None)
    q1, s1 = torch.empty(700, d, device="cuda", dtype=F8), torch.empty(700, vp.fp8_blocks(d), device="cuda")
    vp.vp_rms_forward_fp8(*few, w, 1e-6, q1, s1, None, None)
    assert torch.equal(q[tail].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[tail], s1)
    del q, s, y
    dx, dw = x, torch.empty(d, device="cuda", dtype=torch.bfloat16)         # the gradient over the input, which z has replaced
    ws = torch.empty(vp.vp_rms_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    vp.vp_rms_backward(r, None, z, w, rstd, dx, dw, ws)
    dx1 = torch.empty_like(few[0])
    vp.vp_rms_backward(few[1], None, z1, w, rs1, dx1, None, None)
    assert torch.equal(dx[tail], dx1) and torch.isfinite(dw.float()).all()


def test_quantize_blocks():
    rows, d = 270000, 8192
    w = fill(rows, d)
    q, s = vp.quantize_blocks_fp8(w)
    first = (rows - 1) // 128 * 128 - 256                                   # whole blocks, and the last ragged one
    q1, s1 = vp.quantize_blocks_fp8(w[first:])
    assert torch.equal(q[first:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[first // 128:], s1)


@pytest.mark.parametrize("T", [5, 100])
def test_token_logp(T):
    V, d = 270000, 8192
    W = fill(V, d).mul_(0.02)
    H = fill(T, d, seed=3)
    tokens = torch.arange(V - T, V, device="cuda", dtype=torch.int32)
    W[V - 3] = H[0] * 0.1                                                   # the first token's best is far behind 2^31
    out = vp.token_log_probs(H, W, tokens, top_k=3)
    ref = orc.token_logp(H[:4], W, tokens[:4], 1.0)
    e_x = (d / 16 + 16) * 2.0 ** -23 * (H[:4].double().abs() @ W.double().abs().mT).amax(1)
    ent = ref["entropy"]
    stat = 2.0 ** -20 * (4 + ent)
    assert ((out.logp[:4].double() - ref["logp"]).abs() <= 2 * e_x + stat + 2.0 ** -22 * ref["logp"].abs()).all()
    assert ((out.entropy[:4].double() - ent).abs() <= (2 * e_x + stat) * (1 + ent)).all()
    assert int(out.top_ids[0, 0]) == V - 3
    del ref
    wq, ws = vp.quantize_blocks_fp8(W)
    hq, hs = vp.rms_norm_fp8(H)
    got = vp.token_log_probs_fp8(hq, hs, wq, ws, tokens, top_k=1)
    assert int(got.top_ids[0, 0]) == V - 3
    last = wq[V - 64 - V % 128:].double() * orc.spread_blocks(ws, V, d)[V - 64 - V % 128:]
    x = (hq.double() * orc.spread_columns(hs, d)) @ last.mT
    want = x[:, -1] - x[:, -2]                                              # the difference of two log probabilities is that of two logits
    a = vp.token_log_probs_fp8(hq, hs, wq, ws, torch.full((T,), V - 1, device="cuda")).logp
    b = vp.token_log_probs_fp8(hq, hs, wq, ws, torch.full((T,), V - 2, device="cuda")).logp
    sizes = (hq.double() * orc.spread_columns(hs, d)).abs() @ last[-2:].abs().mT
    e_x = (d / 32 + 16 + 3 * d / 128) * 2.0 ** -23 * sizes.amax(1)
    assert ((((a - b).double() - want).abs()) <= 2 * e_x + 2.0 ** -21 * (a.abs() + b.abs())).all()


@pytest.mark.parametrize("rows,d", [(270000, 8192), (2100000, 1024), (1940000, 1111), (34000000, 64), (130000, 17000)])
def test_rms_norm_gradients_from_the_last_rows_alone(rows, d):
    """An upstream gradient that is zero up to the last 700 rows, and the sum's: dx is dz before them, and dweight what those rows give, against
    float64.  Every term but 700 is an exact zero, so the sums are off by (700 + 64) 2^-24 sum|dy zh|; zh by e_rs = (k / 2 + 6) 2^-24 with
    k = d / 256 + 40."""
    assert rows * d > 1 << 31
    tail = slice(rows - 700, rows)
    z, dz, w = fill(rows, d), fill(rows, d, seed=1), 1 + 0.2 * fill(d, seed=2).float()
    dy = torch.zeros_like(z)
    dy[tail] = fill(700, d, seed=3)
    y, rstd = torch.empty_like(z), torch.empty(rows, device="cuda")
    vp.vp_rms_forward(z, None, w, 1e-6, y, None, rstd)
    dx, dw = y.fill_(float("nan")), torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((vp.vp_rms_workspace_bytes(rows, d),), 255, dtype=torch.uint8, device="cuda")
    vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)
    assert torch.equal(dx[:rows - 700], dz[:rows - 700])
    alone, dw1 = torch.empty(700, d, device="cuda", dtype=torch.bfloat16), torch.empty_like(dw)
    vp.vp_rms_backward(dy[tail].clone(), dz[tail].clone(), z[tail].clone(), w, rstd[tail].clone(), alone, dw1, ws)
    assert torch.equal(dx[tail], alone)
    zh = z[tail].double()
    zh = zh / torch.sqrt((zh * zh).mean(1, keepdim=True) + 1e-6)
    terms = dy[tail].double() * zh
    e = 2.0 ** -24 * ((700 + 64) + (d / 256 + 40) / 2 + 6)
    for got in (dw, dw1):
        assert ((got.double() - terms.sum(0)).abs() <= e * terms.abs().sum(0)).all()
