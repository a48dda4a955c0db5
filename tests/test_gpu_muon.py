"""GPU parity of the Muon update and of the orthogonalisation alone against the float64 oracle on the same inputs.

Tolerance of the orthogonalised update O (relative Frobenius error): every step rounds X, A and B to fp16, a relative error of
2^-12 / sqrt(3) of each entry in the mean square; the three roundings of the five steps add in quadrature to 5.5e-4 of the
result, and the iteration carries a perturbation on to its result with a factor of at most 8 over the spectra used here
(its steepest part, the plateau's edge).  5e-3 bounds that.  Then (fp32 arithmetic, u = 2^-24)
    p   lr scale 5e-3 |O|_F + 4 u |p|_F,   entries: lr scale 8e-2 max(|O|, rms O) + 4 u |p|
    m   4 u (|mu m| + |g|) entry by entry
and w is the bf16 rounding of the new p, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import training_ops_oracle as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TOL_O = 5e-3
COEFFS = orc.MUON_COEFFS


def gradient(batch, rows, cols, seed, dtype=torch.float32, spikes=3):
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(batch, rows, cols, generator=gen, dtype=torch.float64)
    if spikes:
        g += 0.3 * torch.randn(batch, rows, spikes, generator=gen, dtype=torch.float64) @ torch.randn(batch, spikes, cols, generator=gen, dtype=torch.float64)
    return (1e-3 * g).to(dtype).cuda()


def workspace(batch, rows, cols, extra=0):
    n = vp.muon_workspace_bytes(batch, rows, cols)
    assert n > 0
    return torch.full((n + extra,), 255, dtype=torch.uint8, device="cuda")


def orth(g, dtype=torch.float32, **kw):
    b, r, c = (1, *g.shape) if g.dim() == 2 else g.shape
    o = torch.full(g.shape, float("nan"), dtype=dtype, device="cuda")
    ws = workspace(b, r, c)
    vp.muon_orthogonalize(g, o, ws, **kw)
    assert vp.muon_device_status(ws) == 0
    return o


def rel(a, b):
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


def oracle(g, **kw):
    return np.stack([orc.orthogonalize(x, **kw) for x in g.double().cpu().numpy()])


SHAPES = [(1, 1, 1), (1, 1, 7), (2, 9, 1), (1, 2, 3), (1, 64, 64), (1, 63, 65), (2, 128, 256), (1, 256, 128), (1, 256, 256), (1, 257, 300),
          (3, 300, 257), (1, 500, 1203), (1, 1203, 500), (1, 512, 512), (1, 640, 640), (1, 1030, 130), (40, 48, 60), (2, 385, 769),
          (1, 129, 2100), (9, 200, 450), (5, 100, 500), (2, 512, 90), (3, 200, 250), (2, 250, 140), (170, 30, 20), (1, 128, 513), (1, 257, 257)]


@pytest.mark.parametrize("batch,rows,cols", SHAPES)
def test_orthogonalize_matches_oracle(batch, rows, cols):
    g = gradient(batch, rows, cols, seed=rows * 3 + cols)
    o = orth(g).double().cpu().numpy()
    ref = oracle(g)
    for i in range(batch):
        assert rel(o[i], ref[i]) <= TOL_O
        assert np.abs(o[i] - ref[i]).max() <= 8e-2 * max(np.sqrt((ref[i] ** 2).mean()), np.abs(ref[i]).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
def test_types_and_in_place(dtype, out):
    g = gradient(2, 190, 310, seed=1, dtype=dtype)
    ref = oracle(g)
    o = orth(g, out)
    half = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12, torch.float32: 0.0}[out]
    assert rel(o.double().cpu().numpy(), ref) <= TOL_O + half
    if out is dtype:
        h = g.clone()
        vp.muon_orthogonalize(h, h, workspace(2, 190, 310))
        assert torch.equal(h, o)
    one = orth(g[1], out)                                               # [rows, cols] without a batch dimension
    assert one.shape == g[1].shape and torch.equal(one, o[1])


def test_spectra():
    """Exactly known singular values: f applied five times to each of them."""
    rng = np.random.default_rng(0)
    q1, _ = np.linalg.qr(rng.standard_normal((150, 150)))
    q2, _ = np.linalg.qr(rng.standard_normal((400, 150)))
    a, b, c = COEFFS
    for s in (np.ones(150), np.linspace(0.05, 1, 150), np.where(np.arange(150) < 10, 1.0, 0.0)):
        g = (q1 * s) @ q2.T
        o = orth(torch.from_numpy(g).float().cuda()[None])[0].double().cpu().numpy()
        t = s / np.linalg.norm(s)
        x = [np.linalg.norm(t)]                                         # |X_k|_F
        for _ in range(5):
            t = a * t + b * t ** 3 + c * t ** 5
            x.append(np.linalg.norm(t))
        # Directions that the gradient lacks: what rounding puts there at X_k grows by `a` in each step that is left.  One
        # rounding makes X_0, three (A, B, X) make each later X_k; the last stays in fp32, its A and B count once more.
        noise = [485.0 / 3.4445 ** k * (1 if k == 0 else 3 ** 0.5) * 2.0 ** -12 / 3 ** 0.5 * x[k] / x[5] for k in range(6)]
        tol = TOL_O if (s > 0).all() else 2 * float(np.sqrt(np.sum(np.square(noise))))
        assert rel(o, (q1 * t) @ q2.T) <= tol


def test_scale_invariance_zero_and_tiny_gradients():
    g = gradient(1, 130, 200, seed=4)
    o = orth(g)
    # powers of two change nothing but exponents
    for e in (-40, 30):
        assert torch.equal(orth(g * 2.0 ** e, eps=0.0), o)
    z = torch.zeros(2, 70, 90, device="cuda")
    z[1] = gradient(1, 70, 90, seed=5)[0]
    o = orth(z)
    assert not o[0].any() and rel(o[1:].double().cpu().numpy(), oracle(z[1:])) <= TOL_O
    # a norm below eps: X_0 = U / eps stays small, as the definition says
    t = gradient(1, 60, 60, seed=6) * 1e-9
    ref = oracle(t)
    assert np.linalg.norm(t.cpu().numpy()) < 1e-7
    assert rel(orth(t).double().cpu().numpy(), ref) <= TOL_O


def test_bad_values_stay_in_their_matrix():
    g = gradient(4, 140, 180, seed=7)
    ref = orth(g)
    g[1, 3, 5] = float("nan")
    g[2, 0, 0] = float("inf")
    o = orth(g)
    assert torch.equal(o[0], ref[0]) and torch.equal(o[3], ref[3])
    assert torch.isnan(o[1]).any() and torch.isnan(o[2]).any()


def test_steps_and_coefficients():
    g = gradient(2, 210, 330, seed=8)
    for steps in (1, 2, 3, 7):
        assert rel(orth(g, steps=steps).double().cpu().numpy(), oracle(g, steps=steps)) <= TOL_O
    # coefficients of their own in each step, cubic ones (c = 0) among them: 1.5 x - 0.5 x^3 converges to the orthogonal factor
    ks = [(4.0848, -6.8946, 2.9270), (3.9505, -6.3029, 2.6377), (3.7418, -5.5913, 2.3037), (2.8769, -3.1427, 1.2046), (2.8366, -3.0525, 1.2012)]
    assert rel(orth(g, coeffs=ks).double().cpu().numpy(), oracle(g, coeffs=ks)) <= TOL_O
    cubic = [(1.5, -0.5, 0.0)] * 18
    o = orth(g, coeffs=cubic, steps=18).double().cpu().numpy()
    assert rel(o, oracle(g, coeffs=cubic, steps=18)) <= TOL_O
    assert np.abs(o[0] @ o[0].T - np.eye(210)).max() <= 2e-2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 256, 256), (3, 130, 70), (2, 70, 130), (1, 300, 301), (1, 999, 250)])
def test_step_matches_oracle(batch, rows, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    p = 0.02 * torch.randn(batch, rows, cols, generator=gen, device="cuda")
    m = 2e-3 * torch.randn(batch, rows, cols, generator=gen, device="cuda")
    w = torch.full(p.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lr, mu, wd, scale = 0.02, 0.95, 0.1, vp.muon_rms_scale(rows, cols)
    for k, nesterov in enumerate((True, False, True)):
        g = gradient(batch, rows, cols, seed=31 * k + rows, dtype=dtype)
        p0, m0, g0 = (t.double().cpu().numpy() for t in (p, m, g))
        ws = workspace(batch, rows, cols)
        vp.muon_step(p, m, g, w, lr, mu, wd, scale, ws, nesterov=nesterov)
        assert vp.muon_device_status(ws) == 0
        assert torch.equal(w, p.to(torch.bfloat16))
        for i in range(batch):
            rp, rm, ro = orc.muon_step(p0[i], m0[i], g0[i], lr, mu, nesterov, wd, scale)
            err = np.abs(p[i].double().cpu().numpy() - rp)
            assert np.linalg.norm(err) <= lr * scale * TOL_O * np.linalg.norm(ro) + 4 * U * np.linalg.norm(p0[i])
            big = np.maximum(np.abs(ro), np.sqrt((ro ** 2).mean()))
            assert np.all(err <= lr * scale * 8e-2 * big + 4 * U * np.abs(p0[i]))
            assert np.all(np.abs(m[i].double().cpu().numpy() - rm) <= 4 * U * (np.abs(mu * m0[i]) + np.abs(g0[i])))


def test_step_without_working_weight_and_frozen_learning_rate():
    g = gradient(1, 90, 140, seed=2)
    p, m = torch.randn(1, 90, 140, device="cuda"), torch.zeros(1, 90, 140, device="cuda")
    p2, m2, w2 = p.clone(), m.clone(), torch.empty(1, 90, 140, dtype=torch.bfloat16, device="cuda")
    vp.muon_step(p, m, g, None, 1e-2, 0.9, 0.0, 1.0, workspace(1, 90, 140))
    vp.muon_step(p2, m2, g, w2, 1e-2, 0.9, 0.0, 1.0, workspace(1, 90, 140))
    assert torch.equal(p, p2) and torch.equal(m, m2)
    before = p.clone()
    vp.muon_step(p, m, g, None, 0.0, 0.9, 0.5, 1.0, workspace(1, 90, 140))
    assert torch.equal(p, before) and not torch.equal(m, m2)             # lr = 0: the master stays, the momentum moves
    # momentum 0 and a zero momentum buffer: the orthogonalised gradient itself
    p3, m3 = torch.zeros_like(p), torch.zeros_like(m)
    vp.muon_step(p3, m3, g, None, 1.0, 0.0, 0.0, 1.0, workspace(1, 90, 140))
    assert torch.equal(m3, g) and rel(-p3.double().cpu().numpy(), oracle(g)) <= TOL_O


def test_repeats_streams_and_graph():
    g = gradient(3, 700, 900, seed=9)
    ref = orth(g)
    for _ in range(3):
        assert torch.equal(orth(g), ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, ws = torch.empty_like(ref), workspace(3, 700, 900)
    torch.cuda.synchronize()
    vp.muon_orthogonalize(g, o, ws, stream=s)
    s.synchronize()
    assert torch.equal(o, ref)
    # two calls in flight on two streams, each with its own workspace
    outs = [torch.empty_like(ref) for _ in range(2)]
    wss = [workspace(3, 700, 900) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for q, oo, w in zip(streams, outs, wss):
            vp.muon_orthogonalize(g, oo, w, stream=q)
    torch.cuda.synchronize()
    assert all(torch.equal(t, ref) for t in outs) and all(vp.muon_device_status(w) == 0 for w in wss)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vp.muon_orthogonalize(g, o, ws)
    o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, ref)


def test_memory_beyond_the_workspace_is_untouched():
    n = vp.muon_workspace_bytes(2, 100, 333)
    ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    g = gradient(2, 100, 333, seed=1)
    o = torch.full((4, 100, 333), 5.0, device="cuda")
    vp.muon_orthogonalize(g, o[1:3], ws[:n])
    torch.cuda.synchronize()
    assert (ws[n:] == 77).all() and (o[0] == 5).all() and (o[3] == 5).all()


def test_refusals_and_empty_calls():
    g = gradient(1, 64, 96, seed=1)
    o, ws = torch.empty_like(g), workspace(1, 64, 96, extra=1024)
    p, m = torch.zeros_like(g), torch.zeros_like(g)
    for call, err in [(lambda: vp.muon_orthogonalize(g.cpu(), o, ws), TypeError), (lambda: vp.muon_orthogonalize(g.double(), o, ws), TypeError),
                      (lambda: vp.muon_orthogonalize(g, o[:, :32], ws), ValueError), (lambda: vp.muon_orthogonalize(g[0, 0], o[0, 0], ws), ValueError),
                      (lambda: vp.muon_orthogonalize(g.transpose(1, 2), o.transpose(1, 2), ws), ValueError),
                      (lambda: vp.muon_orthogonalize(g, o, ws, coeffs=[(1, 2, 3)] * 4), ValueError),
                      (lambda: vp.muon_step(p.half(), m, g, None, 0.1, 0.9, 0.0, 1.0, ws), TypeError),
                      (lambda: vp.muon_step(p, m[:, :1], g, None, 0.1, 0.9, 0.0, 1.0, ws), ValueError),
                      (lambda: vp.muon_step(p, m, g, p, 0.1, 0.9, 0.0, 1.0, ws), TypeError)]:
        with pytest.raises(err):
            call()
    for call, code in [(lambda: vp.muon_orthogonalize(g, o, ws, steps=0), 1), (lambda: vp.muon_orthogonalize(g, o, ws, steps=33), 1),
                       (lambda: vp.muon_orthogonalize(g, o, ws, eps=-1.0), 1), (lambda: vp.muon_orthogonalize(g, o, ws[:1024]), 3),
                       (lambda: vp.muon_orthogonalize(g, o, ws[128:]), 2), (lambda: vp.muon_orthogonalize(g, o, ws, coeffs=(9.0, 1.0, 1.0)), 2),
                       (lambda: vp.muon_orthogonalize(g, o, ws, coeffs=(float("nan"), 0.0, 0.0)), 2),
                       (lambda: vp.muon_step(p, m, g, None, 0.1, 1.0, 0.0, 1.0, ws), 1),
                       (lambda: vp.muon_step(p, m, g, None, float("inf"), 0.9, 0.0, 1.0, ws), 1)]:
        with pytest.raises(vp.VpceError) as ei:
            call()
        assert ei.value.code == code
    assert vp.muon_workspace_bytes(1, -1, 4) == 0 and vp.muon_workspace_bytes(1 << 20, 4, 4) == 0
    e = torch.empty(0, 5, 5, device="cuda")
    vp.muon_orthogonalize(e, e.clone(), ws)
    e = torch.empty(2, 0, 5, device="cuda")
    vp.muon_orthogonalize(e, e.clone(), ws)
