"""A policy step with an entropy bonus and an 8-bit reference head, with the operators as they are used together.

A small policy (embedding, one residual block, final RMS norm of the residual stream, vocabulary projection) answers prompts and takes
steps on its answers:

    generate    hidden of one new token per answer -> rms_norm -> token_log_probs (alternatives) -> a draw among them
    reference   rms_norm_fp8 -> token_log_probs_fp8 with the head quantised once (quantize_blocks_fp8): no gradient, half the bytes
    step        rms_norm (with the residual) -> token_log_probs (log probability and entropy) -> policy_loss - bonus * entropy -> backward

    python examples/entropy_policy_step.py --steps 4
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_14306_b200 as vp  # noqa: E402


class Policy:
    """bf16 weights; the block's output is added to the residual stream by the final norm."""

    def __init__(self, vocab: int = 512, d: int = 128, seed: int = 0, device: str = "cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape, std):
            return (std * torch.randn(*shape, generator=gen, device=device)).to(torch.bfloat16).requires_grad_(True)

        self.weights = {"embedding": weight(vocab, d, std=1.0), "block": weight(d, d, std=d ** -0.5),
                        "norm": torch.ones(d, dtype=torch.bfloat16, device=device, requires_grad=True), "head": weight(vocab, d, std=2 * d ** -0.5)}

    def stream(self, tokens: torch.Tensor):
        """(the block's output, the residual stream) at `tokens` [T]."""
        residual = torch.nn.functional.embedding(tokens, self.weights["embedding"])
        return torch.tanh(residual @ self.weights["block"].t()), residual

    def score(self, tokens: torch.Tensor, targets: torch.Tensor, temperature: float = 1.0, top_k: int = 0) -> "vp.TokenLogProbs":
        out, residual = self.stream(tokens)
        hidden, _ = vp.rms_norm(out, self.weights["norm"], residual)
        return vp.token_log_probs(hidden, self.weights["head"], targets, top_k=top_k, temperature=temperature, block_v=256)


class Reference:
    """A frozen copy whose head works on 8-bit operands."""

    def __init__(self, policy: Policy):
        self.policy = Policy.__new__(Policy)
        self.policy.weights = {k: w.detach().clone() for k, w in policy.weights.items()}
        self.head, self.head_scales = vp.quantize_blocks_fp8(self.policy.weights["head"])

    @torch.no_grad()
    def logp(self, tokens: torch.Tensor, targets: torch.Tensor, temperature: float = 1.0) -> torch.Tensor:
        out, residual = self.policy.stream(tokens)
        hidden, scales, _ = vp.rms_norm_fp8(out, self.policy.weights["norm"], residual)
        return vp.token_log_probs_fp8(hidden, scales, self.head, self.head_scales, targets, temperature=temperature).logp


@torch.no_grad()
def generate(policy: Policy, prompts: torch.Tensor, length: int, temperature: float, top_k: int, noise: torch.Tensor):
    """Answers of `length` tokens to one-token prompts [n], each token drawn among the top_k alternatives; noise [length, n, top_k] in
    (0, 1).  Returns the tokens that were read and those that followed, both [n, length]."""
    read, following, now = [], [], prompts
    for step in range(length):
        out, residual = policy.stream(now)
        hidden, _ = vp.rms_norm(out, policy.weights["norm"], residual)
        alternatives = vp.token_log_probs(hidden, policy.weights["head"], top_k=top_k, temperature=temperature)
        # the largest of log probability plus Gumbel noise is a draw from the (renormalised) alternatives
        pick = (alternatives.top_logp - torch.log(-torch.log(noise[step]))).argmax(1, keepdim=True)
        chosen = alternatives.top_ids.gather(1, pick)[:, 0].long()
        read.append(now)
        following.append(chosen)
        now = chosen
    return torch.stack(read, 1), torch.stack(following, 1)


def policy_steps(steps: int = 4, n: int = 24, length: int = 17, temperature: float = 0.9, bonus: float = 0.01, lr: float = 0.05, seed: int = 0):
    """Steps on one batch of generated answers; returns the losses and the gradients of the last step by weight."""
    policy = Policy(seed=seed)
    reference = Reference(policy)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    prompts = torch.randint(0, 512, (n,), generator=gen, device="cuda")
    noise = torch.rand(length, n, 8, generator=gen, device="cuda").clamp_(1e-6, 1 - 1e-6)
    read, following = (t.reshape(-1) for t in generate(policy, prompts, length, temperature, 8, noise))
    offsets = torch.arange(0, n * length + 1, length, device="cuda")
    advantages = torch.randn(n, generator=gen, device="cuda")
    with torch.no_grad():
        old = policy.score(read, following, temperature).logp
    ref = reference.logp(read, following, temperature)
    losses = []
    for _ in range(steps):
        for w in policy.weights.values():
            w.grad = None
        scored = policy.score(read, following, temperature)
        loss, _ = vp.policy_loss(scored.logp, old, advantages, offsets, ref_logp=ref, kl_coef=0.02)
        loss = loss - bonus * scored.entropy.mean()
        loss.backward()
        with torch.no_grad():
            for w in policy.weights.values():
                w -= (lr * w.grad.float()).to(w.dtype)
        losses.append(float(loss.detach()))
    return losses, {k: w.grad for k, w in policy.weights.items()}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=4)
    losses, grads = policy_steps(ap.parse_args().steps)
    for i, loss in enumerate(losses):
        print(f"step {i}: loss {loss:+.5f}")
    print("gradient norms: " + ", ".join(f"{k} {float(g.float().norm()):.4f}" for k, g in grads.items()))


if __name__ == "__main__":
    main()
