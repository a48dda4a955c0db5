"""Policy and preference loss at the edges of what the C entries accept, where the paths of small and large calls meet, and
where the terms are small differences of large numbers.  Oracle and helpers are those of test_gpu_sequence_loss."""
import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
import test_gpu_sequence_loss as seq

pytestmark = pytest.mark.gpu


def library():
    vp.vp_policy_loss_workspace_bytes(0, 0)                              # binds the signatures
    return vp.load_library()


def stream():
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------------------------------------ calls without sequences
@pytest.mark.parametrize("T", [0, 1, 300, 8192, 8193])
def test_no_sequences_and_null_offsets(T):
    """n_seqs == 0 needs no offsets: statistics and gradients are 0 in the one-launch and the three-launch path."""
    lib = library()
    x = torch.randn(max(T, 1), device="cuda")
    d = torch.full((T + 8,), 9.0, device="cuda")
    s4, s3 = torch.full((4,), 9.0, device="cuda"), torch.full((3,), 9.0, device="cuda")
    ws = torch.full((vp.vp_policy_loss_workspace_bytes(T, 0),), 255, dtype=torch.uint8, device="cuda")
    for per_token in (0, 1):
        for aggregate in (0, 1):
            d.fill_(9.0), s4.fill_(9.0)
            args = (x.data_ptr(), x.data_ptr(), x.data_ptr(), x.data_ptr() if per_token else None, per_token, None, None, T, 0, 0.2,
                    0.2, 0.1, aggregate)
            assert lib.vp_policy_loss(*args, s4.data_ptr(), d.data_ptr(), None, ws.data_ptr(), ws.numel(), stream()) == 0
            torch.cuda.synchronize()
            assert not s4.any() and not d[:T].any() and (d[T:] == 9).all()
            d.fill_(9.0)
            assert lib.vp_policy_loss_backward(*args, d.data_ptr(), None, ws.data_ptr(), ws.numel(), stream()) == 0
            torch.cuda.synchronize()
            assert not d[:T].any() and (d[T:] == 9).all()
    for kind in (0, 1):
        d.fill_(9.0), s3.fill_(9.0)
        assert lib.vp_preference_loss(x.data_ptr(), None, None, None, T, 0, 0.1, 0.0, 0.0, kind, 0, s3.data_ptr(), None, d.data_ptr(), None,
                                      ws.data_ptr(), ws.numel(), stream()) == 0
        torch.cuda.synchronize()
        assert not s3.any() and not d[:T].any() and (d[T:] == 9).all()


# ------------------------------------------------------------------------------------------------ sequences without tokens
@pytest.mark.parametrize("n", [2, 1024, 1026, 5000])
def test_sequences_but_no_tokens(n):
    """T == 0 with few and with many sequences: every sequence is empty.  The policy loss is 0; the preference loss is the loss
    of D = 0, exactly (one fp32 rounding of log 2 and its like)."""
    f = torch.empty(0, device="cuda")
    off = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    adv = torch.randn(n, device="cuda")
    for aggregate in ("token_mean", "seq_mean"):
        stats = torch.full((4,), 9.0, device="cuda")
        ws = torch.full((vp.vp_policy_loss_workspace_bytes(0, n),), 255, dtype=torch.uint8, device="cuda")
        vp.vp_policy_loss(f, f, f, adv, None, off, 0.2, 0.2, 0.1, aggregate, stats, f.clone(), ws, adv_per_token=False)
        vp.vp_policy_loss_backward(f, f, f, adv, None, off, 0.2, 0.2, 0.1, aggregate, f.clone(), ws, adv_per_token=False)
        assert not stats.any()
    for kind, loss in (("sigmoid", np.log(2.0)), ("ipo", 25.0)):
        stats, rewards = torch.full((3,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        ws = torch.full((vp.vp_preference_loss_workspace_bytes(0, n // 2),), 255, dtype=torch.uint8, device="cuda")
        vp.vp_preference_loss(f, None, None, off, 0.1, 0.0, 0.0, kind, True, stats, rewards, f.clone(), ws)
        vp.vp_preference_loss_backward(None, off, f.clone(), ws)
        got = stats.cpu().numpy()
        assert abs(got[0] - loss) <= 2.0 ** -22 * loss and got[1] == 0 and got[2] == 0
        assert not rewards.any()


# ------------------------------------------------------------------------------------------------ KL near the reference
U = 2.0 ** -24


def kl_terms(logp, ref):
    """q, e^q - q - 1 and e^q - 1 in float64 of the fp32 inputs (at |q| >= 1e-7 the difference keeps eight digits there)."""
    q = ref.astype(np.float64) - logp.astype(np.float64)
    return q, np.expm1(q) - q, np.expm1(q)


def run_policy(logp, old, ref, adv, off, kl_coef, aggregate):
    T, n = len(logp), len(off) - 1
    dev = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (logp, old, ref, adv)]
    stats, d = torch.full((4,), float("nan"), device="cuda"), torch.full((T,), float("nan"), device="cuda")
    ws = torch.full((vp.vp_policy_loss_workspace_bytes(T, n),), 255, dtype=torch.uint8, device="cuda")
    args = (*dev, None, torch.tensor(off, dtype=torch.int64, device="cuda"), 0.2, 0.2, kl_coef, aggregate)
    vp.vp_policy_loss(*args, stats, d, ws, adv_per_token=True)
    again = torch.full_like(d, float("nan"))
    vp.vp_policy_loss_backward(*args, again, ws, adv_per_token=True)
    assert torch.equal(d, again)                                         # the gradient call repeats the joint call's bits
    return stats.cpu().numpy().astype(np.float64), d.cpu().numpy().astype(np.float64)


def test_kl_of_single_tokens():
    """One token, so the statistic is its estimate.  Relative error: at most 35 u of the form (1 ulp of e^q over
    the result, at |q| = 1/8 or beyond), q's rounding (2 + |q|) u, the mean's 2 u."""
    logp = np.array([-1.0], np.float32)
    for size in (1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.1, 0.12499, 0.12501, 0.3, 1.0, 5.0):
        for sign in (1.0, -1.0):
            ref = (logp + np.float32(sign * size)).astype(np.float32)
            q, kl, _ = kl_terms(logp, ref)
            stats, _ = run_policy(logp, logp, ref, np.zeros(1, np.float32), [0, 1], 0.125, "token_mean")
            tol = (40 + abs(q[0])) * U * kl[0]
            assert stats[1] >= 0 and abs(stats[1] - kl[0]) <= tol, (size, sign, stats[1], kl[0])
            assert abs(stats[0] - 0.125 * kl[0]) <= tol


@pytest.mark.parametrize("aggregate", ["token_mean", "seq_mean"])
@pytest.mark.parametrize("lens", [[700, 0, 41, 759], [9000, 1, 11000]])
@pytest.mark.parametrize("spread", [1e-4, 1e-3, 3e-2, 0.3, 1.0])
def test_kl_near_the_reference(spread, lens, aggregate):
    """A policy that has just left its reference: mean and gradient keep their digits, whatever the distance.  With advantages
    of 0 the loss is the KL term alone.  All terms have one sign, so errors are relative:
        mean       (37 + |q|) u per token and (T / 1024 + 40) u of the sums, 4 u around them
        gradient   2 u of e^q - 1, (1 + |q|) u of q, one each for kl_coef x, its weight, their product; 4 u spare"""
    rng = np.random.default_rng(3)
    off = np.concatenate([[0], np.cumsum(lens)])
    T = int(off[-1])
    logp = -np.abs(rng.standard_normal(T) * 1.5).astype(np.float32) - np.float32(0.5)
    ref = (logp + rng.standard_normal(T) * spread).astype(np.float32)
    q, kl, x = kl_terms(logp, ref)
    stats, grad = run_policy(logp, logp, ref, np.zeros(T, np.float32), off, 0.125, aggregate)
    biggest = np.abs(q).max()
    rel = (37 + biggest + T / 1024 + 40 + 4) * U
    if aggregate == "token_mean":
        w = np.full(T, 1.0 / T)
    else:
        have = [n for n in lens if n]
        w = np.concatenate([np.full(n, 1.0 / n / len(have)) for n in have])
    assert stats[1] >= 0 and abs(stats[1] - kl.mean()) <= rel * kl.mean()
    assert abs(stats[0] - 0.125 * (w * kl).sum()) <= rel * 0.125 * (w * kl).sum()
    want = -0.125 * w * x
    assert np.all(np.abs(grad - want) <= (10 + np.abs(q)) * U * np.abs(want))


# ------------------------------------------------------------------------------------------------ close pairs of large sums
@pytest.mark.parametrize("n", [4000, 100000])
def test_difference_of_large_sums(n):
    """Sequences of n tokens of -1 - 2^-10 and the like, without a reference: sums near -n whose difference is a fraction of
    their fp32 spacing.  All values are multiples of 2^-10 and a tile's sums (up to 2^13 tokens of size under 2) fit fp32
    exactly, so D is known exactly and what follows is rounded a few times: stats 4 u, slopes (beta, z, the curve, one rounding
    of the weight) 10 u."""
    step = 2.0 ** -10
    a, b = np.full(n, -1.0 - step), np.full(n, -1.0 - step)
    a[n // 3] += step                                                    # D = 2^-10 in the first pair
    c, d = b.copy(), b.copy()
    c[7] -= 3 * step                                                     # D = -3 * 2^-10 in the second
    logp = np.concatenate([a, c, b, d]).astype(np.float32)               # preferred ones first
    off = torch.arange(5, dtype=torch.int64, device="cuda") * n
    x = torch.from_numpy(logp).cuda()
    ws = torch.full((vp.vp_preference_loss_workspace_bytes(4 * n, 2),), 255, dtype=torch.uint8, device="cuda")
    stats, rewards, g = torch.empty(3, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4 * n, device="cuda")
    D = np.array([step, -3 * step])
    for kind, beta, margin, average in (("sigmoid", 64.0, 0.5, False), ("ipo", 128.0, 0.0, False), ("ipo", 1024.0, 0.0, True)):
        vp.vp_preference_loss(x, None, None, off, beta, margin, 0.0, kind, average, stats, rewards, g, ws)
        diff, count = (D / n, n) if average else (D, 1)
        if kind == "sigmoid":
            z = beta * diff - margin
            loss, slope = np.log1p(np.exp(-z)).mean(), -beta / (1 + np.exp(z))
        else:
            loss, slope = ((diff - 0.5 / beta) ** 2).mean(), 2 * (diff - 0.5 / beta)
        got = stats.cpu().numpy().astype(np.float64)
        # with `average` the means are rounded to double at their own size, 2^-53 of 1: that is beta 2^-52 / |D| of D, far below u
        assert abs(got[0] - loss) <= 8 * U * loss and got[1] == 0.5
        assert abs(got[2] - beta * diff.mean()) <= 4 * U * abs(beta * diff.mean())
        w = g.view(4, n).cpu().numpy().astype(np.float64)
        for i in range(2):
            for row, sign in ((i, 1.0), (2 + i, -1.0)):
                want = sign * slope[i] / 2 / count
                assert np.all(np.abs(w[row] - want) <= 10 * U * abs(want)), (kind, i, w[row][0], want)


# ------------------------------------------------------------------------------------------------ a batch in parts
@pytest.mark.parametrize("aggregate", ["token_mean", "seq_mean"])
def test_parts_of_a_batch_add_up_to_the_whole(aggregate):
    """Each part's loss times its share of the valid tokens (sequences), back-propagated, is the whole batch's gradient.  Both
    sides round their weight and two products, 4 u each, and the share 2 u: 10 u element by element."""
    rng = np.random.default_rng(4)
    lens = [300, 0, 41, 500, 7, 260]
    off = np.concatenate([[0], np.cumsum(lens)])
    T = int(off[-1])
    logp = torch.from_numpy(-np.abs(rng.standard_normal(T)).astype(np.float32)).cuda()
    old, mask = logp + 0.1 * torch.randn(T, device="cuda"), torch.from_numpy(rng.random(T) < 0.7).cuda()
    adv, ref = torch.randn(len(lens), device="cuda"), logp - 0.05

    def share(lo, hi):
        if aggregate == "token_mean":
            return mask[off[lo]:off[hi]].sum().float()
        return torch.tensor(float(sum(bool(mask[off[s]:off[s + 1]].any()) for s in range(lo, hi))), device="cuda")

    def loss(x, lo, hi):
        t = slice(int(off[lo]), int(off[hi]))
        o = torch.from_numpy(off[lo:hi + 1] - off[lo]).cuda()
        return vp.policy_loss(x[t], old[t], adv[lo:hi], o, mask=mask[t], ref_logp=ref[t], kl_coef=0.1, aggregate=aggregate)[0]

    whole, parts = (logp.clone().requires_grad_(True) for _ in range(2))
    full = loss(whole, 0, 6)
    full.backward()
    N, total = share(0, 6), 0.0
    for lo, hi in ((0, 3), (3, 6)):
        part = loss(parts, lo, hi) * (share(lo, hi) / N)
        part.backward()
        total += float(part.detach())
    assert torch.all((parts.grad - whole.grad).abs() <= 10 * U * whole.grad.abs())
    # sums: (T / 1024 + 40) u of the mean term, 8 u around them, on both sides; a term is at most 2 |A| (ratios below 2)
    assert abs(total - float(full.detach())) <= 2 * (T / 1024 + 48) * U * 2 * float(adv.abs().max())


# ------------------------------------------------------------------------------------------------ where the paths meet
SWITCH = [[8192], [8193], [8191, 1], [8000, 193], [1] * 1023 + [0], [1] * 1025, [8] * 1024, [8] * 1024 + [0], [8] * 1023 + [0, 9]]


@pytest.mark.parametrize("i", range(len(SWITCH)))
def test_both_sides_of_the_switch_between_the_paths(i):
    """One launch serves up to 8192 tokens in up to 1024 sequences; both sides of either limit, against the oracle."""
    off, T, logp, old, ref, mask, adv, adv_seq = seq.make(SWITCH[i], seed=40 + i)
    for aggregate in ("token_mean", "seq_mean"):
        seq.check_policy(off, T, logp, old, ref, mask, adv, 0.05, aggregate, True)
        seq.check_policy(off, T, logp, old, None, None, adv_seq, 0.0, aggregate, False, upstream=0.5)
    if len(SWITCH[i]) % 2 == 0:
        seq.check_preference(off, T, logp, ref, mask, 0.1, 0.2, 0.05, "sigmoid", False)
        seq.check_preference(off, T, logp, ref, mask, 0.1, 0.0, 0.0, "ipo", True)


@pytest.mark.parametrize("n_seqs", [1024, 1025])
def test_same_tokens_on_both_paths(n_seqs):
    """An empty sequence at the end is the difference between the paths and none to the result: they agree to the oracle's bounds
    twice over (token by token 2 (8 + |q| ...) u, here 64 u)."""
    lens = [7] * 1024
    off, T, logp, old, ref, mask, adv, _ = seq.make(lens, seed=3)
    base = seq.policy(off, T, logp, old, ref, mask, adv, 0.1, "token_mean", True)
    more = seq.policy(np.concatenate([off] + [[T]] * (n_seqs - 1024)), T, logp, old, ref, mask, adv, 0.1, "token_mean", True)
    assert np.all(np.abs(base[0] - more[0]) <= 128 * U * np.maximum(np.abs(base[0]), 1.0))
    assert np.all(np.abs(base[1] - more[1]) <= 64 * U * np.abs(base[1]))


# ------------------------------------------------------------------------------------------------ two streams
def test_early_started_launches_on_two_streams():
    """The later launches of a large call start before the one in front of them has ended.  Calls of both losses in flight on two
    streams, back to back on each, give what they give alone."""
    rng = np.random.default_rng(6)
    off = torch.tensor([0, 20000, 20001, 45000, 70000], device="cuda")
    T = 70000
    logp = torch.from_numpy(-np.abs(rng.standard_normal(T)).astype(np.float32)).cuda()
    old, ref, adv = logp + 0.1 * torch.randn(T, device="cuda"), logp - 0.05, torch.randn(T, device="cuda")
    mask = torch.from_numpy(rng.random(T) < 0.7).cuda()

    def policy_call(out, stream=None):
        vp.vp_policy_loss(logp, old, ref, adv, mask, off, 0.2, 0.2, 0.1, "seq_mean", *out, adv_per_token=True, stream=stream)

    def preference_call(out, stream=None):
        vp.vp_preference_loss(logp, ref, mask, off, 0.1, 0.0, 0.0, "ipo", True, out[0], None, *out[1:], stream=stream)

    def buffers(stats):
        ws = max(vp.vp_policy_loss_workspace_bytes(T, 4), vp.vp_preference_loss_workspace_bytes(T, 2))
        return torch.zeros(stats, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(ws, dtype=torch.uint8, device="cuda")

    want = buffers(4), buffers(3)
    policy_call(want[0]), preference_call(want[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(buffers(4), buffers(3)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (a, b) in zip(streams, got):
            policy_call(a, s), preference_call(b, s)
    torch.cuda.synchronize()
    for pair in got:
        for g, w in zip(pair, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
