"""The operators from the residual stream to log probabilities as they are used together: residual and RMS norm, log probabilities with
entropy, policy loss, backward, and an 8-bit reference; against the same chain in float64 through torch's own differentiation.

Tolerance: the chain rounds to bf16 at the residual sum, the norm's output, the residual strip of the head's backward pass and every
gradient that is handed on (2^-9 each, at random), some of them twice: 2e-2 in the Frobenius norm of each weight's gradient, 1e-2 in the
loss (its terms are of order 1)."""
import os
import sys

import pytest
import torch

import paper_2609_14306_b200 as vp
from oracle import head_ops_oracle as orc

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import entropy_policy_step as ex  # noqa: E402


def test_example_runs_and_gives_gradients():
    losses, grads = ex.policy_steps(steps=3)
    assert all(map(lambda v: v == v and abs(v) < 1e3, losses))
    assert all(torch.isfinite(g).all() and float(g.float().norm()) > 0 for g in grads.values())


def test_generated_tokens_are_alternatives():
    policy = ex.Policy(seed=3)
    prompts = torch.arange(5, device="cuda")
    noise = torch.rand(4, 5, 3, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").clamp_(1e-6, 1 - 1e-6)
    read, following = ex.generate(policy, prompts, 4, 0.7, 3, noise)
    scored = policy.score(read.reshape(-1), following.reshape(-1), 0.7, top_k=3)
    assert (scored.top_ids.long() == following.reshape(-1, 1)).any(1).all()
    at = (scored.top_ids.long() == following.reshape(-1, 1)).float().argmax(1, keepdim=True)
    # the logit of the given token and that of the alternative are the same number
    assert torch.equal(scored.top_logp.gather(1, at)[:, 0], scored.logp)


def test_chain_against_float64():
    policy = ex.Policy(seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    T, temperature, bonus = 300, 0.9, 0.05
    read, following = (torch.randint(0, 512, (T,), generator=gen, device="cuda") for _ in range(2))
    offsets = torch.tensor([0, 100, 101, 300], device="cuda")
    adv = torch.randn(3, generator=gen, device="cuda")
    ref = ex.Reference(policy).logp(read, following, temperature)
    with torch.no_grad():
        old = policy.score(read, following, temperature).logp + 0.05 * torch.randn(T, generator=gen, device="cuda")
    scored = policy.score(read, following, temperature)
    loss, _ = vp.policy_loss(scored.logp, old, adv, offsets, ref_logp=ref, kl_coef=0.1)
    loss = loss - bonus * scored.entropy.mean()
    loss.backward()

    w = {k: v.detach().double().requires_grad_(True) for k, v in policy.weights.items()}
    residual = w["embedding"][read]
    z = torch.tanh(residual @ w["block"].t()) + residual
    y = z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-6) * w["norm"]
    logq = torch.log_softmax(y @ w["head"].t() / temperature, dim=1)
    logp = logq.gather(1, following[:, None])[:, 0]
    entropy = -(torch.exp(logq) * logq).sum(1)
    a = torch.repeat_interleave(adv.double(), offsets.diff())
    r = torch.exp(logp - old.double())
    q = ref.double() - logp
    want = (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.1 * (torch.exp(q) - q - 1)).mean() - bonus * entropy.mean()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 1e-2
    for k in w:
        got = policy.weights[k].grad.double()
        assert float((got - w[k].grad).norm()) <= 2e-2 * float(w[k].grad.norm()), k


def test_eight_bit_reference_is_near_the_exact_head():
    """8 bits hold 4 significant ones: 2^-4 of each factor at most, at random over 128 columns; log probabilities within 0.2."""
    policy = ex.Policy(seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    read, following = (torch.randint(0, 512, (200,), generator=gen, device="cuda") for _ in range(2))
    with torch.no_grad():
        exact = policy.score(read, following).logp
    assert float((ex.Reference(policy).logp(read, following) - exact).abs().mean()) < 0.2
    # and exactly what the dequantised operands give
    out, residual = policy.stream(read)
    with torch.no_grad():
        q, s, _ = vp.rms_norm_fp8(out, policy.weights["norm"], residual)
    wq, ws = vp.quantize_blocks_fp8(policy.weights["head"])
    got = vp.token_log_probs_fp8(q, s, wq, ws, following)
    want = orc.token_logp(q.double() * orc.spread_columns(s, 128), wq.double() * orc.spread_blocks(ws, 512, 128), following, 1.0)
    assert float((got.logp.double() - want["logp"]).abs().max()) < 1e-4
