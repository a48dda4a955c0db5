"""GPU parity of the RMS norm (forward, 8-bit output, backward) against the float64 definition on the same inputs.

Tolerances.  With u = 2^-24 and k = d / 256 + 40 (an upper bound on the additions that one value goes through in the sums over a
row, plus the few roundings around them), first-order error bounds of the fp32 arithmetic are
    rstd      relative e_rs = (k / 2 + 4) u               (sum of squares k u, half of it in the root, and its own roundings)
    y         |y| (e_rs + 3 u)
    dx        rstd (|a| (e_rs + 4 u) + |zh| (k u mean|a zh| + |mean(a zh)| (3 e_rs + 8 u))) + u (|dx| + |dz|)
    dg        (rows / 148 + 64) u sum|dy zh| + sum|dy zh| e_rs      (every block adds at least its own share in order)
and each result is rounded once to its type: half an ulp, at most 2^-8 (bf16), 2^-11 (fp16; 2^-25 below its normal range) or 2^-24
relative.  The sum x + r is one rounding of the exact sum of two numbers of the type: in fp32 first (exact or rounded at 24 bits),
then to the type, so its bits are those of torch's float sum rounded.  A scale is max|y| / 448: y's error and two roundings.  8 bits
hold 4 significant ones: q * scale is within 2^-4 of |y|, or half of the smallest step 2^-9 times the scale, plus y's error."""
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}
EPS = 1e-6
F8 = torch.float8_e4m3fn


def within(got, ref, err):
    """Every element of got within err of ref (same NaN places)."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    over = torch.nan_to_num((got - ref).abs() - err, nan=0.0)
    if got.numel():
        at = int(over.argmax())
        assert float(over.max()) <= 0, f"off by {float((got - ref).abs().flatten()[at]):.3e} at {at}, allowed {float(err.flatten()[at]):.3e}"


def rounded(ref, err, dtype):
    return err + HALF_ULP[dtype] * (ref.abs() + err) * 1.001 + TINY[dtype]


def make(rows, d, dtype, wdtype, seed, pad=0, offset=0, n=4):
    """n arrays [rows, d] with `pad` elements between rows, `offset` elements into their storage, and a weight."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def view():
        buf = torch.randn(offset + rows * (d + pad) + 1, generator=gen, device="cuda").to(dtype)
        return buf[offset:offset + rows * (d + pad)].view(rows, d + pad)[:, :d]

    return [view() for _ in range(n)], (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(wdtype)


def nan(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), device="cuda").to(dtype)


def check_forward(x, r, w, eps=EPS, fp8=False):
    rows, d = x.shape
    z = None if r is None else nan(rows, d, dtype=x.dtype)
    rstd = nan(rows)
    want_z = x if r is None else (x.float() + r.float()).to(x.dtype)
    y64, rs64 = orc.rms_norm(want_z, w, eps)
    e_rs = ((d / 256 + 40) / 2 + 4) * U
    e_y = y64.abs() * (e_rs + 3 * U)
    if fp8:
        q, scales = torch.zeros(rows, d, device="cuda").to(F8), nan(rows, vp.fp8_blocks(d))
        vp.vp_rms_forward_fp8(x, r, w, eps, q, scales, z, rstd)
        s64 = orc.group_scales(y64)
        within(scales, s64, s64 * (e_rs + 8 * U))
        spread = orc.spread_columns(scales, d)
        within(q.double() * spread, y64, e_y * 1.1 + torch.maximum(y64.abs() * 2.0 ** -4 * 1.001, spread * 2.0 ** -10))
    else:
        y = nan(rows, d, dtype=x.dtype)
        vp.vp_rms_forward(x, r, w, eps, y, z, rstd)
        within(y, y64, rounded(y64, e_y, x.dtype))
    if r is not None:
        assert torch.equal(z, want_z)
    within(rstd, rs64, rs64 * e_rs)
    return want_z, rstd


def check_backward(dy, dz, z, w, rstd, eps=EPS):
    rows, d = z.shape
    dx, dw = nan(rows, d, dtype=z.dtype), nan(d, dtype=z.dtype if w is None else w.dtype)
    ws = torch.full((vp.vp_rms_workspace_bytes(rows, d),), 255, dtype=torch.uint8, device="cuda")
    vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)
    dx64, dw64 = orc.rms_norm_grad(dy, dz, z, w, eps)
    k = d / 256 + 40
    e_rs = (k / 2 + 4) * U
    _, rs = orc.rms_norm(z, None, eps)
    rs = rs[:, None]
    zh, a = z.double() * rs, dy.double() * (1.0 if w is None else w.double())
    e_dx = rs * (a.abs() * (e_rs + 4 * U) + zh.abs() * (k * U * (a * zh).abs().mean(1, keepdim=True)
                                                        + (a * zh).mean(1, keepdim=True).abs() * (3 * e_rs + 8 * U)))
    e_dx += U * (dx64.abs() + (0 if dz is None else dz.double().abs()))
    within(dx, dx64, rounded(dx64, e_dx, z.dtype))
    terms = (dy.double() * zh).abs().sum(0)
    within(dw, dw64, rounded(dw64, terms * ((rows / 148 + 64) * U + e_rs), dw.dtype))


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float16, torch.float32), (torch.float32, torch.float32)]


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (1, 2880), (5, 7), (64, 64), (33, 255), (300, 256), (17, 257), (700, 1000),
                                    (149, 1111), (37, 2880), (20, 4096), (9, 7168), (6, 8192), (5, 8200), (3, 12288), (2, 20001),
                                    (4, 16384), (3, 16383), (1500, 96), (4001, 64), (777, 128), (2049, 200), (1003, 8), (5, 136)])
def test_matches_definition(rows, d, dtype, wdtype):
    (x, r, dy, dz), w = make(rows, d, dtype, wdtype, seed=rows * 7 + d)
    z, rstd = check_forward(x, r, w)
    check_backward(dy, dz, z, w, rstd)
    check_forward(x, r, w, fp8=True)
    z, rstd = check_forward(x, None, w)
    check_backward(dy, None, x, w, rstd)
    check_forward(x, None, w, fp8=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,d", [(300, 12288), (301, 12289), (150, 14336), (5, 16385), (1200, 5120), (2000, 769)])
def test_widths_at_the_switches_between_kernels(rows, d, dtype):
    (x, r, dy, dz), w = make(rows, d, dtype, torch.float32, seed=d)
    z, rstd = check_forward(x, r, w)
    check_backward(dy, dz, z, w, rstd)
    check_backward(dy, None, z, w, rstd)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,d,pad,offset", [(40, 256, 8, 0), (40, 256, 5, 0), (33, 1000, 24, 3), (65, 2880, 2880, 8), (21, 513, 1, 1),
                                               (300, 3, 0, 1), (50, 1, 2, 0), (7, 20001, 3, 0)])
def test_strides_and_offsets(rows, d, pad, offset, dtype):
    (x, r, dy, dz), w = make(rows, d, dtype, dtype, seed=d + pad, pad=pad, offset=offset)
    z, rstd = check_forward(x, r, w)
    check_forward(x, r, w, fp8=True)
    zs = make(rows, d, dtype, dtype, seed=1, pad=pad + 1, offset=offset, n=1)[0][0]
    zs.copy_(z)
    check_backward(dy, dz, zs, w, rstd)


def test_no_weight():
    (x, r, dy, dz), _ = make(50, 1000, torch.bfloat16, torch.float32, seed=3)
    z, rstd = check_forward(x, r, None)
    dx = nan(50, 1000, dtype=x.dtype)
    vp.vp_rms_backward(dy, dz, z, None, rstd, dx, None, None)
    dx64, _ = orc.rms_norm_grad(dy, dz, z, None, EPS)
    assert float((dx.double() - dx64).norm() / dx64.norm()) < 2.0 ** -8


def test_each_output_may_be_left_out():
    (x, r, dy, dz), w = make(41, 2880, torch.bfloat16, torch.float32, seed=5)
    y, y2, z, rstd = nan(41, 2880, dtype=x.dtype), nan(41, 2880, dtype=x.dtype), nan(41, 2880, dtype=x.dtype), nan(41)
    vp.vp_rms_forward(x, r, w, EPS, y, z, rstd)
    vp.vp_rms_forward(x, r, w, EPS, y2, None, None)
    assert torch.equal(y, y2)
    ws = torch.empty(vp.vp_rms_workspace_bytes(41, 2880), dtype=torch.uint8, device="cuda")
    dx, dw, dx2, dw2 = nan(41, 2880, dtype=x.dtype), nan(2880), nan(41, 2880, dtype=x.dtype), nan(2880)
    vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)
    vp.vp_rms_backward(dy, dz, z, w, rstd, dx2, None, None)
    vp.vp_rms_backward(dy, dz, z, w, rstd, None, dw2, ws)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("rows,d", [(700, 2880), (300, 64), (33, 1001), (5, 20001)])
def test_in_place(rows, d):
    (x, r, dy, dz), w = make(rows, d, torch.bfloat16, torch.bfloat16, seed=d)
    y, z, rstd = nan(rows, d, dtype=x.dtype), nan(rows, d, dtype=x.dtype), nan(rows)
    vp.vp_rms_forward(x, r, w, EPS, y, z, rstd)
    a, b = x.clone(), r.clone()
    vp.vp_rms_forward(a, b, w, EPS, a, b, rstd)             # y over x, the sum over the residual
    assert torch.equal(a, y) and torch.equal(b, z)
    ws = torch.empty(vp.vp_rms_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    dx, dw, dw2 = nan(rows, d, dtype=x.dtype), nan(d, dtype=w.dtype), nan(d, dtype=w.dtype)
    vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)
    for over in (dy, dz):
        u, v = dy.clone(), dz.clone()
        out = u if over is dy else v
        vp.vp_rms_backward(u, v, z, w, rstd, out, dw2, ws)
        assert torch.equal(out, dx) and torch.equal(dw, dw2)


def test_special_values_stay_in_their_row():
    for d in (64, 1000, 2880, 1001):
        (x, r, dy, dz), w = make(6, d, torch.bfloat16, torch.bfloat16, seed=d)
        x[1, 3], x[2, 5], x[4] = float("nan"), float("inf"), 0
        r[4] = 0
        y, z = nan(6, d, dtype=x.dtype), nan(6, d, dtype=x.dtype)
        vp.vp_rms_forward(x, r, w, EPS, y, z, None)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2, 5]) and (y[4] == 0).all()
        assert torch.isfinite(y[[0, 3, 5]].float()).all()
        q, s = torch.zeros(6, d, device="cuda").to(F8), nan(6, vp.fp8_blocks(d))
        vp.vp_rms_forward_fp8(x, r, w, EPS, q, s, None, None)
        assert (s[4] == 1).all() and (q[4].float() == 0).all()              # nothing there: scale 1
        assert torch.isfinite(q[[0, 3, 5]].float()).all() and torch.isfinite(s[[0, 3, 5]]).all()
        assert torch.isnan(q[1].float()).all()


def test_scale_of_tiny_groups_stays_normal():
    x = torch.full((2, 256), 1e-30, device="cuda")
    w = torch.full((256,), 1e-20, device="cuda")                            # y about 1e-40 with eps that keeps the row's size
    q, s = torch.zeros(2, 256, device="cuda").to(F8), nan(2, 2)
    vp.vp_rms_forward_fp8(x, None, w, 1e-20, q, s, None, None)
    assert (s >= 2.0 ** -126).all() and torch.isfinite(q.float()).all()


@pytest.mark.parametrize("d", [64, 2880, 1111, 20001])
def test_repeats_bit_for_bit_and_empty(d):
    (x, r, dy, dz), w = make(2000, d, torch.bfloat16, torch.float32, seed=d)
    outs = []
    for _ in range(2):
        y, z, rstd, dx, dw = nan(2000, d, dtype=x.dtype), nan(2000, d, dtype=x.dtype), nan(2000), nan(2000, d, dtype=x.dtype), nan(d)
        ws = torch.empty(vp.vp_rms_workspace_bytes(2000, d), dtype=torch.uint8, device="cuda")
        vp.vp_rms_forward(x, r, w, EPS, y, z, rstd)
        vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)
        outs.append((y, z, rstd, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    dw.fill_(7)
    vp.vp_rms_backward(dy[:0], dz[:0], z[:0], w, rstd[:0], dx[:0], dw, ws)
    assert (dw == 0).all()
    vp.vp_rms_forward(x[:0], r[:0], w, EPS, y[:0], z[:0], rstd[:0])


def test_autograd_against_differences():
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, r, c, e = (torch.randn(3, 5, 33, generator=gen, device="cuda") for _ in range(4))
    w = (1 + 0.1 * torch.randn(33, generator=gen, device="cuda")).requires_grad_()
    x.requires_grad_(), r.requires_grad_()
    y, z = vp.rms_norm(x, w, r)
    ((y * c).sum() + (z * e).sum()).backward()
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()

    def value(xx, ww):
        zz = xx.double() + r.detach().double()
        return (orc.rms_norm(zz.view(-1, 33), ww, 1e-6)[0].view(zz.shape) * c).sum() + (zz * e).sum()

    for t, g in ((x, x.grad), (w, w.grad)):
        dirn = torch.randn(t.shape, generator=gen, device="cuda").double()
        h = 1e-5
        args = lambda s: (x.detach().double() + s * dirn, w.detach()) if t is x else (x.detach(), w.detach().double() + s * dirn)  # noqa: E731
        diff = (value(*args(h)) - value(*args(-h))) / (2 * h)
        assert abs(float((g.double() * dirn).sum() - diff)) <= 1e-5 * float((g.double().abs() * dirn.abs()).sum())


def test_autograd_partial_upstream_and_layouts():
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(6, 40, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w = torch.ones(40, device="cuda", requires_grad=True)
    # only the sum is used
    xa = x.clone().requires_grad_()
    _, z = vp.rms_norm(xa, w, r)
    z.sum().backward()
    assert (xa.grad == 1).all() and (w.grad == 0).all()
    w.grad = None
    # only y is used, with an expanded upstream gradient, from a transposed input
    xt = x.t().contiguous().t().requires_grad_()
    xc = x.clone().requires_grad_()
    y, _ = vp.rms_norm(xt, w, r)
    y.sum().backward()
    g = w.grad.clone()
    w.grad = None
    y, _ = vp.rms_norm(xc, w, r)
    y.backward(torch.ones_like(y))
    assert torch.equal(xt.grad, xc.grad) and torch.equal(w.grad, g)
    # a frozen input, and a frozen weight
    w.grad = None
    vp.rms_norm(x, w).sum().backward()
    assert w.grad is not None
    xc = x.clone().requires_grad_()
    vp.rms_norm(xc, w.detach()).sum().backward()
    assert xc.grad is not None


def test_second_derivative_raises_and_fp8_has_none():
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(vp.rms_norm(x).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()
    with pytest.raises(RuntimeError, match="no gradient"):
        vp.rms_norm_fp8(x)
    with torch.no_grad():
        q, s = vp.rms_norm_fp8(x.view(2, 2, 32))
    assert q.shape == (2, 2, 32) and s.shape == (2, 2, 1)


def test_refusals():
    x, w = torch.randn(4, 32, device="cuda"), torch.ones(32, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(4, device="cuda")
    with pytest.raises(TypeError):
        vp.vp_rms_forward(x.cpu(), None, w, EPS, y, None, rstd)
    with pytest.raises(TypeError):
        vp.vp_rms_forward(x, None, w.half(), EPS, y, None, rstd)
    with pytest.raises(TypeError):
        vp.vp_rms_forward(x, x.half(), w, EPS, y, None, rstd)
    with pytest.raises(ValueError):
        vp.vp_rms_forward(x, None, w, EPS, y, torch.empty_like(x), rstd)    # a sum without a residual
    with pytest.raises(ValueError):
        vp.vp_rms_forward(x, None, w[:31], EPS, y, None, rstd)
    with pytest.raises(ValueError):
        vp.vp_rms_forward(x.t(), None, None, EPS, torch.empty(32, 4, device="cuda"), None, None)
    with pytest.raises(ValueError):
        vp.rms_norm(x, w, residual=x[:2])
    with pytest.raises(vp.VpceError):
        vp.vp_rms_forward(x, None, w, -1.0, y, None, rstd)
    with pytest.raises(vp.VpceError):
        vp.vp_rms_backward(x, None, x, w, rstd, y, torch.empty_like(w), torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        vp.vp_rms_forward_fp8(x, None, w, EPS, y, torch.empty(4, 1, device="cuda"), None, None)
    with pytest.raises(ValueError):
        vp.vp_rms_forward_fp8(x, None, w, EPS, y.to(F8), torch.empty(4, 2, device="cuda"), None, None)


def test_other_stream_and_graph():
    (x, r, dy, dz), w = make(500, 2880, torch.bfloat16, torch.bfloat16, seed=9)
    y, z, rstd, dx, dw = nan(500, 2880, dtype=x.dtype), nan(500, 2880, dtype=x.dtype), nan(500), nan(500, 2880, dtype=x.dtype), nan(2880, dtype=w.dtype)
    ws = torch.empty(vp.vp_rms_workspace_bytes(500, 2880), dtype=torch.uint8, device="cuda")

    def step():
        vp.vp_rms_forward(x, r, w, EPS, y, z, rstd)
        vp.vp_rms_backward(dy, dz, z, w, rstd, dx, dw, ws)

    step()
    want = [t.clone() for t in (y, z, dx, dw)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, z, dx, dw):
        t.fill_(0)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((y, z, dx, dw), want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y.fill_(0)
        step()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want[0])


@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("shape", [(64, 1024), (4, 16, 1024)])
def test_forward_without_backward_frees_its_memory(shape, with_residual):
    """A graph that is dropped without a backward pass holds nothing afterwards."""
    x, r = (torch.randn(shape, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
    w = torch.ones(shape[-1], device="cuda", requires_grad=True)

    def step():
        vp.rms_norm(x, w, r if with_residual else None)

    step()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for _ in range(4):
        step()
    assert torch.cuda.memory_allocated() == before


def test_backward_refuses_a_sum_that_was_written_to():
    x, r = (torch.randn(8, 256, device="cuda", requires_grad=True) for _ in range(2))
    y, z = vp.rms_norm(x, None, r)
    with torch.no_grad():
        z.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
