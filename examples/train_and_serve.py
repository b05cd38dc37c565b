"""A vocabulary head's life on one GPU: sample from it, learn from the samples, bring it to 4 bits, serve it.

A toy policy: one embedding per prompt as the hidden state and a head W [V, D] over the vocabulary.  Each round samples a token
per prompt (sip_sample), rewards those of a favoured set, scores the tokens under the head (sip_xent_forward), takes the
gradient of the advantage-weighted loss (sip_xent_backward), bounds it (sip_grad_clip) and steps.  At the end the head is
quantised (sip_head_quantize) and decodes from its 4-bit codes (sip_head_logits -> sip_sample).

    python examples/train_and_serve.py [--rounds 30] [--prompts 512] [--vocab 32000] [--width 1024]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2506_22033_amd as sip  # noqa: E402


def sample(logits, seed, step, temperature=1.0):
    t = torch.full((logits.shape[0],), temperature, device=logits.device)
    ids, _, logprob = sip.sip_sample(logits, {"temperature": t}, None, None, seed, step, 0)
    return ids, logprob[:, 0]


def run(rounds=30, prompts=512, vocab=32000, width=1024, seed=0, rate=20.0, group=128):
    """(reward of the first and of the last round, reward from the 4-bit head, its largest difference in log-probability)."""
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(seed)
    hidden = torch.randn(prompts, width, generator=g, device=dev).bfloat16()
    weight32 = torch.randn(vocab, width, generator=g, device=dev) / width ** 0.5
    favoured = torch.rand(vocab, generator=g, device=dev) < 0.1
    weight = weight32.bfloat16()
    grad = torch.empty_like(weight)
    workspace = torch.empty(sip.sip_xent_workspace_bytes(prompts, vocab, width, True), dtype=torch.uint8, device=dev)
    table = sip.GradTable([grad])                      # clipped in place
    stride = (vocab + 7) // 8 * 8                      # rows that the sampler takes
    logits = torch.empty(prompts, stride, device=dev)[:, :vocab]
    rewards = []
    for step in range(rounds):
        torch.mm(hidden.float(), weight.float().t(), out=logits)
        ids, logprob = sample(logits, seed, step)
        reward = favoured[ids.long()].float()
        rewards.append(float(reward.mean()))
        advantage = reward - reward.mean()
        loss, lse = sip.sip_xent_forward(hidden, weight, ids, workspace=workspace)
        # what the sampler reported and what the head says of the same tokens
        assert float((loss + logprob).abs().max()) < 1e-3
        sip.sip_xent_backward(hidden, weight, ids, loss, lse, advantage, 1.0 / prompts, grad_weight=grad,
                              want_hidden=False, workspace=workspace)
        sip.sip_grad_clip(table, 1.0)
        weight32 -= rate * grad.float()
        weight.copy_(weight32)

    codes, scales, zeros = sip.sip_head_quantize(weight, group)
    served = sip.sip_head_logits(hidden, codes, scales, zeros)
    ids, logprob = sample(served, seed, rounds)
    loss, _ = sip.sip_xent_forward(hidden, weight, ids, workspace=workspace)
    return rewards[0], rewards[-1], float(favoured[ids.long()].float().mean()), float((loss + logprob).abs().max())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rounds", 30), ("prompts", 512), ("vocab", 32000), ("width", 1024)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    first, last, served, off = run(a.rounds, a.prompts, a.vocab, a.width)
    print(f"reward: first round {first:.3f}, last {last:.3f}, from the 4-bit head {served:.3f}; "
          f"its log-probabilities are off by at most {off:.3f}")


if __name__ == "__main__":
    main()
