"""GPU parity of layer norm (forward and backward) against the float64 oracle on the same inputs.

Tolerances.  With u = 2^-24 and k = d / 256 + 40 (an upper bound on the additions that one value goes through in the sums over
a row, plus the few roundings around them), first-order error bounds of the fp32 arithmetic are
    mean      e_mu = k u mean|x|                 rstd     relative (k / 2 + 8) u + eps-rounding (in the 8)
    xh        e_xh = rstd e_mu + |xh| (k / 2 + 8) u
    y         |g| e_xh + 8 u (|xh g| + |b|)
    dx        rstd (k u mean|a| + |xh| (k u mean|a xh| + mean(|a| e_xh)) + |mean(a xh)| e_xh + 8 u (|a| + |mean a| + |xh mean(a xh)|))
              + |dx| (k / 2 + 8) u
    dg, db    sums over rows: (rows / 148 + 64) u sum|term| + sum(|dy| e_xh)      (every block adds at least its own share in order)
and each result is rounded once to its type: half an ulp, at most 2^-8 (bf16), 2^-11 (fp16; 2^-25 below its normal range) or 2^-24
relative.  mean(.) here are over the row, from the oracle's values."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import training_ops_oracle as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}
EPS = 1e-5


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def bounds(x, dy, g, b, eps):
    """First-order error bounds (before the final rounding) of y, mean, rstd, dx, dg, db."""
    rows, d = x.shape
    k = d / 256 + 40
    _, mean, rstd = orc.layer_norm(x, None, None, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    ga = np.ones(d) if g is None else np.abs(g)
    ba = np.zeros(d) if b is None else np.abs(b)
    e_mu = k * U * np.abs(x).mean(1)
    # a row whose spread is no larger than its mean's rounding: the variance then carries (mean error)^2 as well
    e_rs = (k / 2 + 8) * U + 0.5 * (e_mu * rstd) ** 2
    e_xh = (rstd * e_mu)[:, None] + np.abs(xh) * e_rs[:, None]
    out = {"y": ga * e_xh + 8 * U * (np.abs(xh) * ga + ba), "mean": e_mu, "rstd": rstd * e_rs}
    if dy is not None:
        a = dy * (1.0 if g is None else g)
        ma, mx = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
        dx = rstd[:, None] * (a - ma - xh * mx)
        e_mx = k * U * np.abs(a * xh).mean(1, keepdims=True) + (np.abs(a) * e_xh).mean(1, keepdims=True)
        out["dx"] = rstd[:, None] * (k * U * np.abs(a).mean(1, keepdims=True) + np.abs(xh) * e_mx + np.abs(mx) * e_xh
                                     + 8 * U * (np.abs(a) + np.abs(ma) + np.abs(xh * mx))) + np.abs(dx) * e_rs[:, None]
        kr = (rows / 148 + 64) * U
        out["dg"] = kr * np.abs(dy * xh).sum(0) + (np.abs(dy) * e_xh).sum(0)
        out["db"] = kr * np.abs(dy).sum(0)
    return out


def close(got, ref, err, dtype):
    got = f64(got)
    tol = err + HALF_ULP[dtype] * (np.abs(ref) + err) * 1.001 + TINY[dtype]
    worst = np.max((np.abs(got - ref) - tol) / np.maximum(tol, 1e-300)) if got.size else -1.0
    assert worst <= 0, f"{worst + 1:.2f} times the tolerance"


def make(rows, d, dtype, wdtype, seed, row_pad=0, offset=0):
    """x and dy as views with `row_pad` elements between rows, `offset` elements into their storage."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def view():
        buf = torch.randn(offset + rows * (d + row_pad) + 1, generator=gen, device="cuda").to(dtype)
        return buf[offset:offset + rows * (d + row_pad)].view(rows, d + row_pad)[:, :d]

    x, dy = view(), view()
    x.mul_(1.5).add_(0.25)
    g = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(wdtype)
    b = (0.3 * torch.randn(d, generator=gen, device="cuda")).to(wdtype)
    return x, dy, g, b


def run_both(x, dy, g, b, eps=EPS):
    rows, d = x.shape
    y = torch.full((rows, d), float("nan"), dtype=x.dtype, device="cuda")
    mean, rstd = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    vp.vp_ln_forward(x, g, b, eps, y, mean, rstd)
    wdt = x.dtype if g is None and b is None else (g if g is not None else b).dtype
    dx = torch.full((rows, d), float("nan"), dtype=x.dtype, device="cuda")
    dg, db = torch.full((d,), float("nan"), dtype=wdt, device="cuda"), torch.full((d,), float("nan"), dtype=wdt, device="cuda")
    ws = torch.full((vp.vp_ln_workspace_bytes(rows, d),), 255, dtype=torch.uint8, device="cuda")
    vp.vp_ln_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
    return y, mean, rstd, dx, dg, db


def check(x, dy, g, b, eps=EPS):
    y, mean, rstd, dx, dg, db = run_both(x, dy, g, b, eps)
    x6, dy6, g6, b6 = f64(x), f64(dy), f64(g), f64(b)
    e = bounds(x6, dy6, g6, b6, eps)
    ry, rm, rr = orc.layer_norm(x6, g6, b6, eps)
    rdx, rdg, rdb = orc.layer_norm_grad(dy6, x6, g6, eps)
    close(y, ry, e["y"], x.dtype)
    close(mean, rm, e["mean"], torch.float32)
    close(rstd, rr, e["rstd"], torch.float32)
    close(dx, rdx, e["dx"], x.dtype)
    close(dg, rdg, e["dg"], dg.dtype)
    close(db, rdb, e["db"], db.dtype)


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float16, torch.float32), (torch.float32, torch.float32)]


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (1, 2880), (5, 7), (64, 64), (33, 255), (300, 256), (17, 257), (700, 1000),
                                    (149, 1111), (37, 2880), (20, 4096), (9, 7168), (6, 8192), (5, 8200), (3, 12288), (2, 20001), (4, 16384), (3, 16383),
                                    (1500, 96), (4001, 64), (777, 128), (2049, 200), (1003, 8), (5, 256)])
def test_matches_oracle(rows, d, dtype, wdtype):
    check(*make(rows, d, dtype, wdtype, seed=rows * 7 + d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,d,pad,offset", [(40, 256, 8, 0), (40, 256, 5, 0), (33, 1000, 24, 3), (65, 2880, 2880, 8), (21, 513, 1, 1),
                                               (12, 7168, 1, 0), (3, 9001, 4, 2)])
def test_row_strides_and_alignments(rows, d, pad, offset, dtype):
    check(*make(rows, d, dtype, torch.float32, seed=d + pad, row_pad=pad, offset=offset))


@pytest.mark.parametrize("rows,d", [(70, 384), (13, 1023), (4, 10000)])
def test_missing_weight_bias_and_outputs(rows, d):
    x, dy, g, b = make(rows, d, torch.bfloat16, torch.bfloat16, seed=5)
    check(x, dy, None, None)
    check(x, dy, g, None)
    check(x, dy, None, b)
    # outputs that are not asked for are not computed; the others do not change
    y, mean, rstd, dx, dg, db = run_both(x, dy, g, b)
    ws = torch.empty(vp.vp_ln_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    for want in [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 0)]:
        outs = [torch.empty_like(t) if w else None for t, w in zip((dx, dg, db), want)]
        vp.vp_ln_backward(dy, x, g, mean, rstd, *outs, ws if want[1] or want[2] else None)
        for o, t in zip(outs, (dx, dg, db)):
            assert o is None or torch.equal(o, t)
    y2 = torch.empty_like(y)
    vp.vp_ln_forward(x, g, b, EPS, y2, None, None)
    assert torch.equal(y, y2)


@pytest.mark.parametrize("rows,d", [(50, 512), (11, 777), (3, 9000)])
def test_in_place(rows, d):
    x, dy, g, b = make(rows, d, torch.float32, torch.float32, seed=9)
    y, mean, rstd, dx, dg, db = run_both(x, dy, g, b)
    x2, dy2 = x.clone(), dy.clone()
    ws = torch.empty(vp.vp_ln_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    vp.vp_ln_backward(dy2, x2, g, mean, rstd, dy2, dg2, db2, ws)
    vp.vp_ln_forward(x2, g, b, EPS, x2, None, None)
    assert torch.equal(dy2, dx) and torch.equal(dg2, dg) and torch.equal(db2, db) and torch.equal(x2, y)


@pytest.mark.parametrize("d", [5, 512, 2880, 9999])
def test_large_common_offset_and_constant_rows(d):
    # a mean 4000 times the spread: the variance of centred values keeps its digits
    x, dy, g, b = make(24, d, torch.float32, torch.float32, seed=d)
    x.add_(4000.0)
    check(x, dy, g, b)
    # constant rows: variance 0, rstd = 1 / sqrt(eps), y = b up to what the mean's rounding leaves
    x[:] = torch.arange(24, device="cuda", dtype=torch.float32)[:, None]
    check(x, dy, g, b)


def test_extreme_values_stay_in_their_rows():
    rows, d = 9, 1000
    x, dy, g, b = make(rows, d, torch.bfloat16, torch.bfloat16, seed=3)
    clean = run_both(x, dy, g, b)
    x[2, 5], x[4, 0], x[7, 999] = float("nan"), float("inf"), -float("inf")
    y, mean, rstd, dx, dg, db = run_both(x, dy, g, b)
    bad = [2, 4, 7]
    good = [r for r in range(rows) if r not in bad]
    for now, then in ((y, clean[0]), (dx, clean[3]), (mean, clean[1]), (rstd, clean[2])):
        assert torch.equal(now[good], then[good])
    assert torch.isnan(y[bad]).all()
    assert torch.isnan(dg).all() and torch.equal(db, clean[5])
    # the largest finite values of the type
    x, dy, g, b = make(6, 640, torch.bfloat16, torch.float32, seed=4)
    x[1] = torch.where(torch.arange(640, device="cuda") % 2 == 0, 1e17, -1e17).to(torch.bfloat16)
    check(x, dy, g, b)


def test_no_rows_and_determinism():
    d = 300
    x = torch.empty(0, d, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    *_, dx, dg, db = run_both(x, x.clone(), g, g)
    assert dx.shape == (0, d) and not dg.any() and not db.any()
    for rows, dd in [(5000, 320), (3000, 1001)]:
        x, dy, g, b = make(rows, dd, torch.bfloat16, torch.float32, seed=1)
        first = run_both(x, dy, g, b)
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(first, run_both(x, dy, g, b)))


def test_more_rows_than_a_grid():
    check(*make(9001, 40, torch.bfloat16, torch.float32, seed=2))
    check(*make(4099, 1160, torch.float16, torch.float16, seed=2))


@pytest.mark.parametrize("d", [6, 40])
def test_gradient_against_differences(d):
    rows, h = 3, 2.0 ** -7
    x, dy, g, b = make(rows, d, torch.float32, torch.float32, seed=d)
    _, _, _, dx, dg, db = run_both(x, dy, g, b)

    def value(xx, gg, bb):
        y = torch.empty_like(xx)
        vp.vp_ln_forward(xx, gg, bb, EPS, y, None, None)
        return float((y.double() * dy.double()).sum())

    def difference(t, at, call):
        plus, minus = t.clone(), t.clone()
        plus[at] += h
        minus[at] -= h
        return (call(plus) - call(minus)) / (2 * h)

    # truncation: h^2 / 6 times a third derivative of order rstd^3 |dy| d; rounding: 2^-22 sum|y dy| / h
    tol = h * h * float(dy.abs().sum()) * 4 + 2.0 ** -22 * float((dy.abs() * 4).sum()) / h
    for r in range(rows):
        for c in range(0, d, 3):
            assert abs(difference(x, (r, c), lambda t: value(t, g, b)) - float(dx[r, c])) <= tol
    for c in range(0, d, 2):
        assert abs(difference(g, (c,), lambda t: value(x, t, b)) - float(dg[c])) <= tol
        assert abs(difference(b, (c,), lambda t: value(x, g, t)) - float(db[c])) <= tol


def test_autograd_shapes_and_expanded_gradient():
    gen = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(4, 7, 96, generator=gen, device="cuda").transpose(0, 1).requires_grad_(True)      # rows are not contiguous in order
    g = torch.randn(96, generator=gen, device="cuda").requires_grad_(True)
    b = torch.randn(96, generator=gen, device="cuda").requires_grad_(True)
    up = torch.randn(96, generator=gen, device="cuda")
    y = vp.layer_norm(x, g, b)
    assert y.shape == x.shape
    (y * up).sum().backward()
    x6 = f64(x).reshape(-1, 96)
    dy6 = np.broadcast_to(f64(up), x6.shape)
    e = bounds(x6, dy6, f64(g), f64(b), EPS)
    rdx, rdg, rdb = orc.layer_norm_grad(dy6, x6, f64(g), EPS)
    close(x.grad.reshape(-1, 96), rdx, e["dx"], torch.float32)
    close(g.grad, rdg, e["dg"], torch.float32)
    close(b.grad, rdb, e["db"], torch.float32)
    # a sum's upstream gradient is one value expanded over the tensor
    g.grad = None
    vp.layer_norm(x.detach(), g).sum().backward()
    rdg = orc.layer_norm_grad(np.ones_like(x6), x6, f64(g), EPS)[1]
    close(g.grad, rdg, bounds(x6, np.ones_like(x6), f64(g), None, EPS)["dg"], torch.float32)
    # no weight at all, and an empty batch
    z = torch.randn(2, 5, device="cuda", requires_grad=True)
    vp.layer_norm(z).square().sum().backward()
    assert torch.isfinite(z.grad).all()
    e0 = torch.empty(0, 96, device="cuda", requires_grad=True)
    g.grad = None
    vp.layer_norm(e0, g, b).sum().backward()
    assert e0.grad.shape == (0, 96) and not g.grad.any()


def test_other_stream_and_graph():
    x, dy, g, b = make(200, 512, torch.bfloat16, torch.float32, seed=8)
    ref = run_both(x, dy, g, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(ref[0])
    vp.vp_ln_forward(x, g, b, EPS, y, None, None, stream=s)
    s.synchronize()
    assert torch.equal(y, ref[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run_both(x, dy, g, b)
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, ref))


def test_refusals():
    x, dy, g, b = make(4, 64, torch.bfloat16, torch.bfloat16, seed=1)
    y, m = torch.empty_like(x), torch.empty(4, device="cuda")
    ws = torch.empty(vp.vp_ln_workspace_bytes(4, 64), dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError):
        vp.vp_ln_forward(x.cpu(), g, b, EPS, y, None, None)
    with pytest.raises(TypeError):
        vp.vp_ln_forward(x.double(), g, b, EPS, y, None, None)
    with pytest.raises(TypeError):
        vp.vp_ln_forward(x, g.half(), None, EPS, y, None, None)
    with pytest.raises(TypeError):
        vp.vp_ln_forward(x, g, b.float(), EPS, y, None, None)
    with pytest.raises(TypeError):
        vp.vp_ln_forward(x, g, b, EPS, y.float(), None, None)
    with pytest.raises(ValueError):
        vp.vp_ln_forward(x, g[:32], b, EPS, y, None, None)
    with pytest.raises(ValueError):
        vp.vp_ln_forward(x, g, b, EPS, y[:3], None, None)
    with pytest.raises(ValueError):
        vp.vp_ln_forward(x.t(), None, None, EPS, torch.empty(64, 4, dtype=x.dtype, device="cuda"), None, None)
    with pytest.raises(ValueError):
        vp.vp_ln_forward(x[:1].expand(4, 64), g, b, EPS, y, None, None)
    with pytest.raises(ValueError):
        vp.vp_ln_forward(x, g, b, EPS, y, m[:3], None)
    with pytest.raises(vp.VpceError) as ei:
        vp.vp_ln_forward(x, g, b, -1.0, y, None, None)
    assert ei.value.code == 1
    with pytest.raises(vp.VpceError) as ei:
        vp.vp_ln_backward(dy, x, g, m, m, None, torch.empty_like(g), None, ws[:-16])
    assert ei.value.code == 3
    with pytest.raises(vp.VpceError) as ei:
        vp.vp_ln_backward(dy, x, g, m, m, None, torch.empty_like(g), None, None)
    assert ei.value.code == 1
    with pytest.raises(TypeError):
        vp.layer_norm(x.cpu())
