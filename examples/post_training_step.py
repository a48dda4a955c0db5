"""A post-training step around the head, with the operators as they are used together.

A small policy (embedding, one trunk matrix, final layer norm, vocabulary projection) takes steps on packed answers:

    hidden = trunk(embedding)  ->  layer_norm  ->  vocab_proj_cross_entropy  (logp = - its per-token loss)
    logp   ->  policy_loss or preference_loss  ->  backward through the head and the norm
    muon_step for the trunk matrix, osadamw_update_device for everything else (fp32 state, bf16 working weights)

    python examples/post_training_step.py --objective policy --steps 8
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_14306_b200 as vp  # noqa: E402


class Policy:
    """bf16 working weights with fp32 masters and optimiser state beside them."""

    def __init__(self, vocab: int, d: int, seed: int = 0, device: str = "cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape, std):
            return std * torch.randn(*shape, generator=gen, device=device)

        self.master = {"embedding": weight(vocab, d, std=1.0), "trunk": weight(d, d, std=d ** -0.5), "norm_w": torch.ones(d, device=device),
                       "norm_b": torch.zeros(d, device=device), "head": weight(vocab, d, std=d ** -0.5)}
        self.work = {k: v.to(torch.bfloat16).requires_grad_(True) for k, v in self.master.items()}
        self.m = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.v = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.muon_ws = torch.empty(vp.muon_workspace_bytes(1, d, d), dtype=torch.uint8, device=device)
        self.t = 0

    def logp(self, tokens: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Log probabilities of `targets` [T] after `tokens` [T] (targets of -100: 0, not looked at by the losses)."""
        w = self.work
        hidden = torch.nn.functional.embedding(tokens, w["embedding"]) @ w["trunk"].t()
        return -vp.vocab_proj_cross_entropy(vp.layer_norm(hidden, w["norm_w"], w["norm_b"]), w["head"], targets, block_v=256)

    def update(self, lr_matrix: float, lr: float, weight_decay: float = 0.01) -> None:
        self.t += 1
        for k, work in self.work.items():
            master, grad = self.master[k], work.grad
            if k == "trunk":
                # the products run on the bf16 gradient; master and momentum stay fp32
                vp.muon_step(master, self.m[k], grad, work.data, lr_matrix, 0.95, weight_decay, vp.muon_rms_scale(*master.shape), self.muon_ws)
            else:
                vp.osadamw_update_device(master.view(-1), self.m[k].view(-1), self.v[k].view(-1), grad.float().view(-1), work.data.view(-1),
                                         lr, 0.9, 0.95, 1e-8, weight_decay, self.t)
            work.grad = None


def batch(vocab: int, n_seqs: int, mean_len: int, seed: int = 0, device: str = "cuda"):
    """Packed ragged answers: tokens, targets (prompts are ignored), mask of the answers' tokens, offsets."""
    gen = torch.Generator().manual_seed(seed)
    lens = torch.randint(mean_len // 2, mean_len * 3 // 2 + 1, (n_seqs,), generator=gen)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(lens, 0)])
    T = int(offsets[-1])
    tokens = torch.randint(0, vocab, (T,), generator=gen)
    position = torch.arange(T) - torch.repeat_interleave(offsets[:-1], lens)
    mask = position >= torch.repeat_interleave(lens // 4, lens)
    targets = torch.where(mask, torch.randint(0, vocab, (T,), generator=gen), torch.tensor(-100))
    return tokens.to(device), targets.to(device), mask.to(device), offsets.to(device)


def policy_steps(steps: int = 8, vocab: int = 512, d: int = 128, n_seqs: int = 16, mean_len: int = 40, seed: int = 0):
    """Steps on one rollout batch; returns the loss of each step (negative: the objective gained) and the last statistics."""
    policy = Policy(vocab, d, seed)
    tokens, targets, mask, offsets = batch(vocab, n_seqs, mean_len, seed)
    with torch.no_grad():
        old = policy.logp(tokens, targets)
    reward = torch.randn(n_seqs, generator=torch.Generator().manual_seed(seed + 1)).cuda()
    advantages = (reward - reward.mean()) / reward.std()
    losses, stats = [], None
    for _ in range(steps):
        loss, stats = vp.policy_loss(policy.logp(tokens, targets), old, advantages, offsets, mask=mask, ref_logp=old, clip_low=0.2,
                                     clip_high=0.28, kl_coef=0.02, aggregate="seq_mean")
        loss.backward()
        policy.update(lr_matrix=2e-3, lr=1e-3)
        losses.append(float(loss.detach()))
    return losses, stats.tolist()


def preference_steps(steps: int = 8, vocab: int = 512, d: int = 128, n_pairs: int = 8, mean_len: int = 40, seed: int = 0):
    """Steps on one batch of pairs; returns the loss of each step and the last statistics."""
    policy = Policy(vocab, d, seed)
    tokens, targets, mask, offsets = batch(vocab, 2 * n_pairs, mean_len, seed)
    with torch.no_grad():
        ref = policy.logp(tokens, targets)
    losses, stats = [], None
    for _ in range(steps):
        loss, stats, _ = vp.preference_loss(policy.logp(tokens, targets), offsets, ref_logp=ref, mask=mask, beta=0.1)
        loss.backward()
        policy.update(lr_matrix=2e-3, lr=1e-3)
        losses.append(float(loss.detach()))
    return losses, stats.tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--objective", choices=("policy", "preference"), default="policy")
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    losses, stats = (policy_steps if a.objective == "policy" else preference_steps)(a.steps)
    for i, loss in enumerate(losses):
        print(f"step {i}: loss {loss:+.5f}")
    names = ("loss", "kl", "clipped", "ratio") if a.objective == "policy" else ("loss", "pairs won", "reward gap")
    print("last step: " + ", ".join(f"{n} {v:.4f}" for n, v in zip(names, stats)))


if __name__ == "__main__":
    main()
