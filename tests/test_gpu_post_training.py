"""The operators around the head together: the example's steps, and one step's gradients against plain PyTorch in float32 on the
same bf16 weights (TOL_GRAD of the head: its gradients' relative Frobenius error; the norm's bf16 output and gradient round two
more times, 2^-9 each, so twice that bound)."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2609_14306_b200 as vp
from vpce_testlib import TOL_GRAD

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import post_training_step as ex  # noqa: E402

pytestmark = pytest.mark.gpu


def test_policy_steps_improve_the_objective():
    losses, stats = ex.policy_steps(steps=8)
    assert abs(losses[0]) < 0.2 and losses[-1] < losses[0] - 0.05       # the first step's ratios are all 1
    assert stats[1] > 0 and 0 < stats[2] < 1 and np.isfinite(stats).all()


def test_preference_steps_separate_the_pairs():
    losses, stats = ex.preference_steps(steps=8)
    assert abs(losses[0] - np.log(2.0)) < 1e-6                           # policy = reference: log 2 exactly
    assert losses[-1] < 0.5 * losses[0] and stats[1] == 1.0 and stats[2] > 0


def test_gradients_through_norm_head_and_loss_match_pytorch():
    policy = ex.Policy(vocab=700, d=96, seed=3)
    tokens, targets, mask, offsets = ex.batch(700, 10, 30, seed=3)
    with torch.no_grad():
        old = policy.logp(tokens, targets) + 0.1 * torch.randn(tokens.numel(), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    adv = torch.randn(10, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    loss, _ = vp.policy_loss(policy.logp(tokens, targets), old, adv, offsets, mask=mask, clip_low=10.0, clip_high=10.0)
    loss.backward()
    w = {k: v.detach().float().requires_grad_(True) for k, v in policy.work.items()}
    hidden = (torch.nn.functional.embedding(tokens, w["embedding"]) @ w["trunk"].t())
    # the same roundings of the activations as in bf16, straight through in the gradient
    hidden = hidden + (hidden.detach().to(torch.bfloat16).float() - hidden.detach())
    h = torch.nn.functional.layer_norm(hidden, (96,), w["norm_w"], w["norm_b"])
    h = h + (h.detach().to(torch.bfloat16).float() - h.detach())
    logp = -torch.nn.functional.cross_entropy(h @ w["head"].t(), targets, ignore_index=-100, reduction="none")
    a = adv[torch.repeat_interleave(torch.arange(10, device="cuda"), offsets.diff())]
    ref = -(torch.exp(logp - old) * a)[mask].mean()
    ref.backward()
    assert abs(float(loss.detach()) - float(ref.detach())) <= 1e-3 * max(1.0, abs(float(ref.detach())))
    for k in w:
        got, want = policy.work[k].grad.float(), w[k].grad
        assert float((got - want).norm() / want.norm()) <= 2 * TOL_GRAD, k
