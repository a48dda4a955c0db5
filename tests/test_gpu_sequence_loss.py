"""GPU parity of the policy loss and the preference loss over packed sequences against the float64 oracle.

Tolerances (u = 2^-24, the unit roundoff of fp32; inputs are fp32 and exact).  r = exp(logp - old): the difference carries
u |logp - old|, the exponential 2 ulp: relative error (|logp - old| + 6) u; likewise e^q with q = ref - logp.  Per token
    e_l    = |A| r (|logp - old| + 8) u + kl_coef (e^q (|q| + 8) + |q| + 4) u
    e_grad = the same with e^q (|q| + 8) + 2
    sums   at most 2 T / 2048 + 40 fp32 additions in a lane and a warp, then double: + (T / 1024 + 40) u mean|term|
Weights (1 / n, 1 / (n S)) are rounded once, products twice more: 4 u relative.  The preference loss sums logp - ref the same
way, with e_s = (T / 1024 + 40) u sum|logp - ref| + u sum(|logp| + |ref|); slopes are formed in double from sums rounded to
fp32, so their error is |d slope / dD| (2 e_s + u |D|...) + 4 u |slope|."""
import math

import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import training_ops_oracle as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LO, HI = 0.2, 0.28


def cuda(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def packed(lens, head=0, tail=0):
    off = head + np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return off, int(off[-1]) + tail


def make(lens, seed, head=0, tail=0, masked=0.3):
    rng = np.random.default_rng(seed)
    off, T = packed(lens, head, tail)
    logp = -np.abs(rng.standard_normal(T) * 1.5).astype(np.float32)
    old = (logp + rng.standard_normal(T) * 0.2).astype(np.float32)
    ref = (logp + rng.standard_normal(T) * 0.1).astype(np.float32)
    # no ratio within 1e-4 of a clip bound: there the fp32 and the float64 comparison may differ
    r = np.exp(logp.astype(np.float64) - old)
    near = (np.abs(r - (1 - LO)) < 1e-4) | (np.abs(r - (1 + HI)) < 1e-4)
    old[near] = logp[near]
    mask = rng.random(T) >= masked
    adv = rng.standard_normal(T).astype(np.float32)
    adv[::11] = 0.0
    adv_seq = rng.standard_normal(len(lens)).astype(np.float32)
    return off, T, logp, old, ref, mask, adv, adv_seq


def policy(off, T, logp, old, ref, mask, adv, kl, agg, per_token, want_grad=True, upstream=None, split=False):
    n = len(off) - 1
    stats = torch.full((4,), float("nan"), device="cuda")
    dlogp = torch.full((T,), float("nan"), device="cuda") if want_grad else None
    ws = torch.full((vp.vp_policy_loss_workspace_bytes(T, n),), 255, dtype=torch.uint8, device="cuda")
    up = None if upstream is None else torch.full((1,), upstream, device="cuda")
    args = (cuda(logp), cuda(old), cuda(ref), cuda(adv), cuda(mask, torch.bool), cuda(off, torch.int64), LO, HI, kl, agg)
    if split:
        vp.vp_policy_loss(*args, stats, None, ws, adv_per_token=per_token)
        vp.vp_policy_loss_backward(*args, dlogp, ws, upstream=up, adv_per_token=per_token)
    else:
        vp.vp_policy_loss(*args, stats, dlogp, ws, upstream=up, adv_per_token=per_token)
    return stats.cpu().numpy().astype(np.float64), None if dlogp is None else dlogp.cpu().numpy().astype(np.float64)


def check_policy(off, T, logp, old, ref, mask, adv, kl, agg, per_token, upstream=1.0):
    stats, grad = policy(off, T, logp, old, ref, mask, adv, kl, agg, per_token, upstream=upstream)
    l6, o6, r6 = (None if a is None else a.astype(np.float64) for a in (logp, old, ref))
    a6 = adv.astype(np.float64)
    loss, rstats, rgrad = orc.policy_loss(l6, o6, r6, a6, per_token, mask, off, LO, HI, kl, agg)
    # error bounds, token by token, over the tokens that count
    lens = np.diff(off)
    A = np.zeros(T)
    inside = np.zeros(T, bool)
    for s, n in enumerate(lens):
        A[off[s]:off[s + 1]] = a6[off[s]:off[s + 1]] if per_token else a6[s]
        inside[off[s]:off[s + 1]] = True
    valid = inside if mask is None else inside & mask
    with np.errstate(all="ignore"):
        x = np.where(valid, l6 - o6, 0.0)
        r = np.exp(x)
        q = np.where(valid, r6 - l6, 0.0) if ref is not None else np.zeros(T)
    k = kl if ref is not None else 0.0
    e_l = np.abs(A) * r * (np.abs(x) + 8) * U + k * (np.exp(q) * (np.abs(q) + 8) + np.abs(q) + 4) * U
    e_g = np.abs(A) * r * (np.abs(x) + 8) * U + k * (np.exp(q) * (np.abs(q) + 8) + 2) * U
    terms = np.abs(A) * np.maximum(r, 1.0) + k * np.abs(np.exp(q) - q - 1)
    nv = max(int(valid.sum()), 1)
    depth = (T / 1024 + 40) * U
    if agg == "token_mean":
        w = valid / nv
    else:
        w = np.zeros(T)
        have = max(sum(1 for s in range(len(lens)) if valid[off[s]:off[s + 1]].any()), 1)
        for s in range(len(lens)):
            v = valid[off[s]:off[s + 1]]
            w[off[s]:off[s + 1]] = v / max(int(v.sum()), 1) / have
    tol = np.array([(w * (e_l + depth * terms)).sum() + 4 * U * abs(rstats[0]),
                    (valid * ((np.exp(q) * (np.abs(q) + 8) + np.abs(q) + 4) * U + depth * np.abs(np.exp(q) - q - 1))).sum() / nv,
                    depth, (valid * r * ((np.abs(x) + 8) * U + depth)).sum() / nv]) + 1e-37
    assert np.all(np.abs(stats - rstats) <= tol), (stats, rstats, tol)
    up = abs(upstream)
    assert np.all(np.abs(grad - upstream * rgrad) <= up * (w * e_g + 4 * U * np.abs(rgrad)) + 1e-37)
    assert not grad[~valid].any()
    return stats, grad


LENS = [[1], [0], [7], [256], [257], [255, 1, 256, 513], [0, 0, 5, 0, 300, 0], [1] * 70, [3000, 2, 1500, 0, 700], [20000],
        list(np.random.default_rng(1).integers(0, 4, 3000)), list(np.random.default_rng(2).integers(0, 900, 140))]


@pytest.mark.parametrize("agg", ["token_mean", "seq_mean"])
@pytest.mark.parametrize("i", range(len(LENS)))
def test_policy_matches_oracle(i, agg):
    off, T, logp, old, ref, mask, adv, adv_seq = make(LENS[i], seed=i)
    check_policy(off, T, logp, old, ref, mask, adv, 0.05, agg, True)
    check_policy(off, T, logp, old, None, None, adv_seq, 0.05, agg, False, upstream=-2.5)


@pytest.mark.parametrize("agg", ["token_mean", "seq_mean"])
def test_policy_tokens_outside_and_garbage_under_the_mask(agg):
    lens = [300, 0, 41, 800, 3]
    off, T, logp, old, ref, mask, adv, adv_seq = make(lens, seed=5, head=17, tail=600)
    mask[off[2]:off[3]] = False                                        # a sequence whose mask leaves nothing
    clean = check_policy(off, T, logp, old, ref, mask, adv, 0.1, agg, True)
    junk = np.array([np.nan, np.inf, -np.inf, -3.4e38, 3.4e38], np.float32)
    dead = np.ones(T, bool)
    for s in range(len(lens)):
        dead[off[s]:off[s + 1]] = ~mask[off[s]:off[s + 1]]
    for i, a in enumerate((logp, old, ref, adv)):
        a[dead] = np.roll(np.resize(junk, int(dead.sum())), i)
    stats, grad = policy(off, T, logp, old, ref, mask, adv, 0.1, agg, True)
    np.testing.assert_array_equal(stats, clean[0])
    np.testing.assert_array_equal(grad, clean[1])
    # nothing valid at all
    stats, grad = policy(off, T, logp, old, ref, np.zeros(T, bool), adv, 0.1, agg, True)
    assert not stats.any() and not grad.any()


def test_policy_clip_boundary_signs_and_extremes():
    # r = 1 exactly with clip bounds of 0: the minimum takes the unclipped term
    T = 6
    z = np.zeros(T, np.float32)
    adv = np.array([1, -1, 2, -2, 0, 3], np.float32)
    off = np.array([0, T])
    stats = torch.empty(4, device="cuda")
    d = torch.empty(T, device="cuda")
    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(T, 1), dtype=torch.uint8, device="cuda")
    vp.vp_policy_loss(cuda(z), cuda(z), None, cuda(adv), None, cuda(off, torch.int64), 0.0, 0.0, 0.0, "token_mean", stats, d, ws)
    np.testing.assert_allclose(d.cpu().numpy(), -adv / T, rtol=4 * U)
    assert stats[2] == 0 and stats[3] == 1
    # ratios that overflow and vanish: clipped where the advantage is positive, unbounded loss where it is negative
    logp = np.array([0, 0, -200, -200, 0, 0], np.float32)
    old = np.array([-200, -200, 0, 0, 0, 0], np.float32)
    adv = np.array([1, -1, 1, -1, 1, 1], np.float32)
    stats, grad = policy(np.array([0, 1, 2, 6]), T, logp, old, None, None, adv, 0.0, "token_mean", True)
    assert stats[0] == np.inf and grad[0] == 0 and grad[1] == np.inf and grad[2] == 0 and grad[3] == 0
    check_policy(np.array([0, 4]), 4, logp[2:], old[2:], None, None, adv[2:], 0.0, "seq_mean", True)


@pytest.mark.parametrize("lens", [[700000], [400000, 0, 1, 299998], [100000] * 8])
def test_policy_long_sequences(lens):
    off, T, logp, old, ref, mask, adv, adv_seq = make(lens, seed=7)
    for agg in ("token_mean", "seq_mean"):
        check_policy(off, T, logp, old, ref, mask, adv, 0.02, agg, True)


def test_split_calls_match_the_joint_call_and_repeat():
    off, T, logp, old, ref, mask, adv, adv_seq = make([500, 0, 3000, 77], seed=3)
    for agg in ("token_mean", "seq_mean"):
        a = policy(off, T, logp, old, ref, mask, adv, 0.1, agg, True, upstream=0.75)
        for _ in range(3):
            b = policy(off, T, logp, old, ref, mask, adv, 0.1, agg, True, upstream=0.75, split=True)
            np.testing.assert_array_equal(a[0], b[0])
            np.testing.assert_array_equal(a[1], b[1])


def test_empty_calls():
    f = torch.empty(0, device="cuda")
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    stats = torch.full((4,), 5.0, device="cuda")
    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(0, 0), dtype=torch.uint8, device="cuda")
    vp.vp_policy_loss(f, f, None, f, None, one, LO, HI, 0.0, "seq_mean", stats, f.clone(), ws)
    assert not stats.any()
    # tokens but no sequence: every gradient is 0
    x = torch.randn(300, device="cuda")
    d = torch.full((300,), 9.0, device="cuda")
    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(300, 0), dtype=torch.uint8, device="cuda")
    vp.vp_policy_loss(x, x, None, x, None, one, LO, HI, 0.0, "token_mean", stats, d, ws)
    assert not stats.any() and not d.any()
    s3 = torch.full((3,), 5.0, device="cuda")
    d.fill_(9.0)
    vp.vp_preference_loss(x, None, None, one, 0.1, 0.0, 0.0, "sigmoid", False, s3, torch.empty(0, device="cuda"), d, ws)
    assert not s3.any() and not d.any()


# ------------------------------------------------------------------------------------------------ preference loss
def preference(off, T, logp, ref, mask, beta, margin, eps, kind, average, upstream=None, split=False):
    n = len(off) - 1
    stats, rewards = torch.full((3,), float("nan"), device="cuda"), torch.full((n,), float("nan"), device="cuda")
    dlogp = torch.full((T,), float("nan"), device="cuda")
    ws = torch.full((vp.vp_preference_loss_workspace_bytes(T, n // 2),), 255, dtype=torch.uint8, device="cuda")
    up = None if upstream is None else torch.full((1,), upstream, device="cuda")
    m, o = cuda(mask, torch.bool), cuda(off, torch.int64)
    vp.vp_preference_loss(cuda(logp), cuda(ref), m, o, beta, margin, eps, kind, average, stats, rewards, None if split else dlogp, ws, upstream=up)
    if split:
        vp.vp_preference_loss_backward(m, o, dlogp, ws, upstream=up)
    return tuple(t.cpu().numpy().astype(np.float64) for t in (stats, rewards, dlogp))


def check_preference(off, T, logp, ref, mask, beta, margin, eps, kind, average, upstream=1.0):
    got = preference(off, T, logp, ref, mask, beta, margin, eps, kind, average, upstream=upstream)
    l6, r6 = logp.astype(np.float64), None if ref is None else ref.astype(np.float64)
    loss, rstats, rrew, rgrad = orc.preference_loss(l6, r6, mask, off, beta, margin, eps, kind, average)
    n, P = len(off) - 1, (len(off) - 1) // 2
    e_s, count = np.zeros(n), np.ones(n)
    for s in range(n):
        v = np.arange(off[s], off[s + 1])
        v = v if mask is None else v[mask[v]]
        r = 0.0 if ref is None else r6[v]
        c = max(len(v), 1) if average else 1
        count[s] = c
        e_s[s] = ((T / 1024 + 40) * U * np.abs(l6[v] - r).sum() + U * (np.abs(l6[v]) + np.abs(r)).sum()) / c
    e_s = e_s + 2 * U * np.abs(rrew / beta)
    assert np.all(np.abs(got[1] - rrew) <= beta * e_s + 2 * U * np.abs(rrew) + 1e-37)
    e_D = e_s[:P] + e_s[P:]
    D = (rrew[:P] - rrew[P:]) / beta
    curve = np.full(P, beta * beta / 4) if kind == "sigmoid" else np.full(P, 2.0)      # largest |d slope / dD|
    slope = np.full(P, beta) if kind == "sigmoid" else 2 * np.abs(D - 0.5 / beta)      # at least |slope|
    for i in range(P):
        for s in (i, P + i):
            t = slice(off[s], off[s + 1])
            tol = abs(upstream) * (curve[i] * e_D[i] / P / count[s] + 6 * U * slope[i] / P / count[s])
            assert np.all(np.abs(got[2][t] - upstream * rgrad[t]) <= tol + 1e-37)
    outside = np.ones(T, bool)
    for s in range(n):
        v = np.arange(off[s], off[s + 1])
        outside[v if mask is None else v[mask[v]]] = False
    assert not got[2][outside].any()
    if P:
        tol = [(slope * e_D).mean() + 4 * U * abs(rstats[0]), 1e-7 + (np.abs(D) <= e_D).mean(), beta * e_D.mean() + 4 * U * np.abs(beta * D).mean()]
        if kind == "ipo":
            tol[0] += (e_D ** 2).mean()
        assert np.all(np.abs(got[0] - rstats) <= np.array(tol) + 1e-37), (got[0], rstats, tol)
    return got


PAIRS = [[1, 1], [5, 0], [0, 0], [256, 257, 1, 700], [300, 0, 4, 2, 2, 900], [1] * 130, list(np.random.default_rng(3).integers(0, 600, 90)),
         list(np.random.default_rng(4).integers(0, 3, 2600))]


@pytest.mark.parametrize("kind,average,beta,margin,eps", [("sigmoid", False, 0.1, 0.0, 0.0), ("sigmoid", True, 2.0, 0.5, 0.1),
                                                          ("ipo", True, 0.1, 0.0, 0.0), ("ipo", False, 0.5, 0.0, 0.0)])
@pytest.mark.parametrize("i", range(len(PAIRS)))
def test_preference_matches_oracle(i, kind, average, beta, margin, eps):
    off, T, logp, old, ref, mask, *_ = make(PAIRS[i], seed=20 + i)
    check_preference(off, T, logp, ref, mask, beta, margin, eps, kind, average)
    check_preference(off, T, logp, None, None, beta, margin, eps, kind, average, upstream=3.0)


def test_preference_garbage_saturation_and_long_pairs():
    lens = [400, 30, 0, 1000]
    off, T, logp, old, ref, mask, *_ = make(lens, seed=9, head=5, tail=300)
    mask[off[1]:off[2]] = False
    clean = check_preference(off, T, logp, ref, mask, 0.1, 0.2, 0.05, "sigmoid", False)
    dead = np.ones(T, bool)
    for s in range(4):
        dead[off[s]:off[s + 1]] = ~mask[off[s]:off[s + 1]]
    logp[dead], ref[dead] = np.nan, -np.inf
    for a, b in zip(clean, preference(off, T, logp, ref, mask, 0.1, 0.2, 0.05, "sigmoid", False)):
        np.testing.assert_array_equal(a, b)
    # |z| far beyond the exponential's range: the loss is linear, the slope saturates, nothing is NaN
    off = np.array([0, 2, 4, 6, 8])
    logp = np.array([-1, -1, -4e4, -4e4, -4e4, -4e4, -1, -1], np.float32)
    stats, rewards, grad = preference(off, 8, logp, None, None, 1.0, 0.0, 0.0, "sigmoid", False)
    np.testing.assert_allclose(stats, [(8e4 - 2) / 2, 0.5, 0.0], rtol=1e-6)
    np.testing.assert_allclose(grad, [0, 0, -0.5, -0.5, 0, 0, 0.5, 0.5], rtol=1e-6)
    off, T, logp, old, ref, mask, *_ = make([350000, 10, 20, 250000], seed=12)
    check_preference(off, T, logp, ref, mask, 0.05, 0.0, 0.0, "sigmoid", True)


def test_preference_split_calls_and_repeats():
    off, T, logp, old, ref, mask, *_ = make([500, 600, 3000, 77], seed=3)
    a = preference(off, T, logp, ref, mask, 0.1, 0.0, 0.0, "sigmoid", False, upstream=0.5)
    for _ in range(3):
        for x, y in zip(a, preference(off, T, logp, ref, mask, 0.1, 0.0, 0.0, "sigmoid", False, upstream=0.5, split=True)):
            np.testing.assert_array_equal(x, y)


# ------------------------------------------------------------------------------------------------ gradients, autograd, refusals
def test_gradients_against_differences():
    """Central differences of the float32 losses in directions over all tokens: truncation h^2 / 6 |third derivative| and
    rounding 2^-22 |loss| / h, both with a factor for the direction's size."""
    off, T, logp, old, ref, mask, adv, adv_seq = make([40, 25, 60, 30], seed=2)
    rng = np.random.default_rng(0)
    h = 2.0 ** -8
    r = np.exp(logp.astype(np.float64) - old)
    free = (np.abs(r - (1 - LO)) > 0.02) & (np.abs(r - (1 + HI)) > 0.02)                  # the kinks stay out of the step
    for agg in ("token_mean", "seq_mean"):
        _, grad = policy(off, T, logp, old, ref, mask, adv, 0.1, agg, True)
        for _ in range(3):
            v = (rng.choice([-1.0, 1.0], T) * free).astype(np.float32)
            up = policy(off, T, logp + np.float32(h) * v, old, ref, mask, adv, 0.1, agg, True, want_grad=False)[0][0]
            dn = policy(off, T, logp - np.float32(h) * v, old, ref, mask, adv, 0.1, agg, True, want_grad=False)[0][0]
            assert abs((up - dn) / (2 * h) - (grad * v).sum()) <= h * h * 4 + 2.0 ** -20 / h
    for kind, average in (("sigmoid", False), ("ipo", True)):
        _, _, grad = preference(off, T, logp, ref, mask, 0.3, 0.1, 0.1, kind, average)
        for _ in range(3):
            v = rng.choice([-1.0, 1.0], T).astype(np.float32) * (0.05 if not average else 1.0)
            v = v.astype(np.float32)
            up, dn = (preference(off, T, (logp + np.float32(s * h) * v), ref, mask, 0.3, 0.1, 0.1, kind, average)[0][0] for s in (1, -1))
            assert abs((up - dn) / (2 * h) - (grad * v).sum()) <= h * h * 4 + 2.0 ** -20 * (1 + abs(up)) / h


def test_autograd_front_ends():
    off, T, logp, old, ref, mask, adv, adv_seq = make([300, 20, 500, 180], seed=6)
    o, m = cuda(off, torch.int64), cuda(mask, torch.bool)
    x = cuda(logp).requires_grad_(True)
    loss, stats = vp.policy_loss(x, cuda(old), cuda(adv_seq), o, mask=m, ref_logp=cuda(ref), clip_low=LO, clip_high=HI, kl_coef=0.1,
                                 aggregate="seq_mean")
    assert not stats.requires_grad
    (3.0 * loss).backward()
    s, g = policy(off, T, logp, old, ref, mask, adv_seq, 0.1, "seq_mean", False, upstream=3.0)
    np.testing.assert_array_equal(x.grad.cpu().numpy(), g.astype(np.float32))
    assert float(loss.detach()) == np.float32(s[0])
    x.grad = None
    loss, stats, rewards = vp.preference_loss(x, o, ref_logp=cuda(ref), mask=m, beta=0.2, kind="ipo", average=True)
    loss.backward()
    s, rw, g = preference(off, T, logp, ref, mask, 0.2, 0.0, 0.0, "ipo", True)
    np.testing.assert_array_equal(x.grad.cpu().numpy(), g.astype(np.float32))
    np.testing.assert_array_equal(rewards.cpu().numpy(), rw.astype(np.float32))


def test_bad_offsets_stay_in_bounds():
    # entries outside [0, T] and out of order: the result is unspecified, every token's gradient is written, nothing else is
    T = 1000
    guard = torch.full((3 * T,), 7.0, device="cuda")
    d = guard[T:2 * T]
    x = torch.randn(T, device="cuda")
    stats = torch.empty(4, device="cuda")
    for off in ([-50, 2000, 10, 900, 5000], [900, 100, 800, 0, 1000], [1000, 1000, 0, 0, 0]):
        d.fill_(float("nan"))
        o = torch.tensor(off, dtype=torch.int64, device="cuda")
        ws = torch.zeros(vp.vp_policy_loss_workspace_bytes(T, 4), dtype=torch.uint8, device="cuda")
        for agg in ("token_mean", "seq_mean"):
            vp.vp_policy_loss(x, x, None, x, None, o, LO, HI, 0.0, agg, stats, d, ws)
            torch.cuda.synchronize()
            assert torch.isfinite(d).all()
            assert (guard[:T] == 7).all() and (guard[2 * T:] == 7).all()


def test_refusals():
    T = 64
    x = torch.randn(T, device="cuda")
    o = torch.tensor([0, 30, 64], dtype=torch.int64, device="cuda")
    stats, d = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(T, 2), dtype=torch.uint8, device="cuda")

    def call(logp=x, old=x, ref=None, adv=x, mask=None, off=o, lo=LO, hi=HI, kl=0.0, agg="token_mean", st=stats, dl=d, w=ws):
        vp.vp_policy_loss(logp, old, ref, adv, mask, off, lo, hi, kl, agg, st, dl, w)

    call()
    for bad, err in [(dict(logp=x.cpu()), TypeError), (dict(logp=x.half()), TypeError), (dict(old=x[:5]), ValueError), (dict(adv=x[:7]), ValueError),
                     (dict(mask=torch.ones(T, device="cuda")), TypeError), (dict(off=o.int()), TypeError), (dict(agg="mean"), ValueError),
                     (dict(st=stats[:3]), ValueError), (dict(logp=torch.randn(2 * T, device="cuda")[::2]), ValueError), (dict(off=o[:0]), ValueError)]:
        with pytest.raises(err):
            call(**bad)
    for bad, code in [(dict(lo=-0.1), 1), (dict(hi=float("nan")), 1), (dict(kl=float("nan")), 1), (dict(w=ws[:-32]), 3), (dict(w=ws[8:]), 2)]:
        with pytest.raises(vp.VpceError) as ei:
            call(**bad)
        assert ei.value.code == code
    s3 = torch.empty(3, device="cuda")

    def pref(off=o, beta=0.1, eps=0.0, kind="sigmoid", w=ws):
        vp.vp_preference_loss(x, None, None, off, beta, 0.0, eps, kind, False, s3, None, d, w)

    pref()
    for bad, err in [(dict(off=torch.tensor([0, 3, 5, 64], dtype=torch.int64, device="cuda")), ValueError), (dict(kind="hinge"), ValueError)]:
        with pytest.raises(err):
            pref(**bad)
    for bad, code in [(dict(beta=0.0), 1), (dict(eps=1.5), 1), (dict(w=ws[:-32]), 3)]:
        with pytest.raises(vp.VpceError) as ei:
            pref(**bad)
        assert ei.value.code == code


@pytest.mark.parametrize("lens", [[700, 0, 41], [30000, 1, 9000]])
def test_graph_and_other_stream(lens):
    off, T, logp, old, ref, mask, adv, adv_seq = make(lens, seed=8)
    t = [cuda(x) for x in (logp, old, ref, adv)]
    m, o = cuda(mask, torch.bool), cuda(off, torch.int64)
    stats, d = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    ws = torch.empty(vp.vp_policy_loss_workspace_bytes(T, len(lens)), dtype=torch.uint8, device="cuda")
    call = lambda **kw: vp.vp_policy_loss(*t, m, o, LO, HI, 0.1, "seq_mean", stats, d, ws, **kw)
    call()
    want = stats.clone(), d.clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):                                    # back to back: a call may not start before the one before it is done
        call(stream=s)
    s.synchronize()
    assert torch.equal(stats, want[0]) and torch.equal(d, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
        twice = d * 2                                     # enqueued right behind: sees the finished gradient
    for _ in range(3):
        stats.zero_(), d.zero_(), twice.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(stats, want[0]) and torch.equal(d, want[1]) and torch.equal(twice, 2 * want[1])
