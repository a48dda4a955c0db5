"""The operators around the head over arrays whose offsets pass 32 bits: more than 2^31 elements."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def release_memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("d", [7168, 7169])
def test_layer_norm(d):
    """A row's result does not depend on where it lies: the last rows equal a call on them alone, bit for bit.  Column sums: the
    sum of calls on parts; each fp32 sum is off by at most (rows / 148 + 64) u of the terms' absolute values, below 2 rows in all
    (dy xh has the mean 0.8 + 0.8 in absolute value, dy 1.2)."""
    rows = (1 << 31) // d + 700
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(rows, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    dy.add_(1.0)
    w, b = torch.randn(d, device="cuda"), torch.randn(d, device="cuda")

    def both(x, dy):
        n = x.shape[0]
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dw, db = torch.empty_like(w), torch.empty_like(b)
        vp.vp_ln_forward(x, w, b, 1e-5, y, mean, rstd)
        vp.vp_ln_backward(dy, x, w, mean, rstd, dx, dw, db, torch.empty(vp.vp_ln_workspace_bytes(n, d), dtype=torch.uint8, device="cuda"))
        return y, dx, dw, db

    y, dx, dw, db = both(x, dy)
    assert x.numel() > 1 << 31
    # parts begin on a 16-byte boundary where the whole does, so that they take the same kernel
    cuts = [0, rows // 3 // 8 * 8, (rows - 600) // 8 * 8, rows]
    parts = [both(x[i:j], dy[i:j]) for i, j in zip(cuts, cuts[1:])]
    for (i, j), part in zip(zip(cuts, cuts[1:]), parts):
        assert torch.equal(y[i:j], part[0]) and torch.equal(dx[i:j], part[1])
    for k, whole in ((2, dw), (3, db)):
        total = sum(p[k].double() for p in parts)
        assert float((whole.double() - total).abs().max()) <= 2 * (rows / 148 + 64) * U * 2 * rows


def test_losses():
    """Gradients around 2^31 and at the end against the formulas in float64; the mean over 2^31 tokens within the additions of a
    lane (524 thousand tokens a tile, 16400 a lane) and the 40 around them."""
    T = (1 << 31) + 12345
    off = torch.tensor([0, 100, (1 << 31) - 5, (1 << 31) + 100, T], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    logp = torch.rand(T, generator=gen, device="cuda").neg_()
    old = torch.rand(T, generator=gen, device="cuda").mul_(0.3).add_(logp).sub_(0.15)
    adv = torch.tensor([1.0, 0.5, -2.0, 3.0], device="cuda")
    depth = (16400 + 40) * U

    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(T, 4), dtype=torch.uint8, device="cuda")
    stats, d = torch.empty(4, device="cuda"), torch.full((T,), float("nan"), device="cuda")
    vp.vp_policy_loss(logp, old, None, adv, None, off, 0.5, 0.5, 0.0, "seq_mean", stats, d, ws)
    lens = off.diff()
    mean_r = 0.0
    for i in range(0, T, 1 << 28):
        mean_r += float((logp[i:i + (1 << 28)] - old[i:i + (1 << 28)]).double().exp_().sum())
    assert abs(float(stats[3]) - mean_r / T) <= depth * mean_r / T and float(stats[2]) == 0
    for lo, hi in ((0, 300), ((1 << 31) - 300, (1 << 31) + 300), (T - 300, T)):
        at = torch.arange(lo, hi, device="cuda")
        s = torch.searchsorted(off[1:].contiguous(), at, right=True)
        r = (logp[lo:hi].double() - old[lo:hi].double()).exp()
        want = -adv[s].double() * r / (4.0 * lens[s].double())
        assert bool(((d[lo:hi].double() - want).abs() <= 12 * U * want.abs()).all())
    assert bool(torch.isfinite(d.view(-1)[:: 4097]).all())

    s3, rewards = torch.empty(3, device="cuda"), torch.empty(4, device="cuda")
    d.fill_(float("nan"))
    vp.vp_preference_loss(logp, old, None, off, 0.1, 0.0, 0.0, "ipo", True, s3, rewards, d, ws)
    means = torch.stack([sum((logp[i:min(i + (1 << 28), int(off[s + 1]))].double() - old[i:min(i + (1 << 28), int(off[s + 1]))].double()).sum()
                             for i in range(int(off[s]), int(off[s + 1]), 1 << 28)) for s in range(4)]) / lens.double()
    # a term is at most 0.15, as is its rounding's share
    assert bool(((rewards.double() - 0.1 * means).abs() <= 0.1 * (depth * 0.15 + 4 * U)).all())
    slope = 2 * (means[:2] - means[2:] - 5.0) / 2
    weight = torch.cat([slope, -slope]) / lens.double()
    for lo, hi in ((0, 300), ((1 << 31) - 300, (1 << 31) + 300), (T - 300, T)):
        s = torch.searchsorted(off[1:].contiguous(), torch.arange(lo, hi, device="cuda"), right=True)
        assert bool(((d[lo:hi].double() - weight[s]).abs() <= (depth * 0.3 + 10 * U) * weight[s].abs()).all())


@pytest.mark.parametrize("batch,rows,cols", [(130, 4096, 4096), (132, 4160, 4000)])
def test_muon(batch, rows, cols):
    """The first, a middle and the last matrix of a batch of more than 2^31 elements against calls on each alone (other tiles,
    perhaps, but the same roundings of the operands: 1e-4 relative is far above what the order of fp32 sums changes and far below
    a wrong matrix)."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    p = torch.randn(batch, rows, cols, generator=gen, device="cuda").mul_(0.02)
    m = torch.randn(batch, rows, cols, generator=gen, device="cuda").mul_(2e-3)
    g = torch.randn(batch, rows, cols, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(1e-3)
    w = torch.empty(batch, rows, cols, device="cuda", dtype=torch.bfloat16)
    assert p.numel() > 1 << 31
    pick = [0, batch // 2, batch - 1]
    before = [(p[i:i + 1].clone(), m[i:i + 1].clone()) for i in pick]
    ws = torch.empty(vp.muon_workspace_bytes(batch, rows, cols), dtype=torch.uint8, device="cuda")
    args = (0.02, 0.95, 0.1, vp.muon_rms_scale(rows, cols))
    vp.muon_step(p, m, g, w, *args, ws)
    assert vp.muon_device_status(ws) == 0
    for i, (q, n) in zip(pick, before):
        old = q.clone()
        vp.muon_step(q, n, g[i:i + 1], None, *args, ws)
        assert torch.equal(n[0], m[i])
        assert float((q[0] - p[i]).norm()) <= 1e-4 * float((q[0] - old[0]).norm())
        assert torch.equal(w[i], p[i].bfloat16())
