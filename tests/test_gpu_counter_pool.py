"""The launches of one backward call share a pool of counters that is zeroed again when it has been used up.  Here the pool runs out
in the middle of what one gradient launch takes (its split tiles' flags, then its tile counter), several times over a call:
25 shards at 8192 tokens, whose gradient launches split 14 tiles.  Every tile has to be written, whichever launch it belongs to."""
import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu


def test_every_tile_is_written_when_the_pool_wraps():
    T, d, V, block_v = 8192, 2880, 201088, 8192
    gen = torch.Generator(device="cuda").manual_seed(0)
    H = torch.randn(T, d, generator=gen, device="cuda").to(torch.bfloat16)
    W = torch.randn(V, d, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(0.02)
    labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    up = torch.randn(T, generator=gen, device="cuda")
    ws = torch.empty(vp.vp_ce_workspace_bytes(T, d, block_v), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    vp.vp_ce_forward(H, W, labels, block_v, -100, loss, lse, T, 0, ws)
    before = vp.vp_ce_set_tail_parts(0)
    try:
        runs = []
        for parts in (0, -1, -1):
            vp.vp_ce_set_tail_parts(parts)
            dH, dW = torch.full_like(H, float("nan")), torch.full((V, d), float("nan"), device="cuda")
            vp.vp_ce_backward(H, W, labels, lse, up, dH, dW, block_v, -100, T, 0, False, ws)
            assert vp.vp_ce_device_status(ws) == 0 and not torch.isnan(dW).any() and not torch.isnan(dH).any()
            runs.append((dH, dW))
        (_, whole), (h1, w1), (h2, w2) = runs
        assert torch.equal(w1, w2) and torch.equal(h1, h2)                  # one order of summation
        # another order of fp32 sums: the same up to 1e-5 in every block of rows
        for a, b in zip(torch.split(w1, 8192), torch.split(whole, 8192)):
            assert float((a - b).norm()) <= 1e-5 * float(b.norm())
    finally:
        vp.vp_ce_set_tail_parts(before)
