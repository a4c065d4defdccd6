"""Language-model workers that train with a clipped policy loss between consensus rounds, on one GPU.

M workers hold replicas of a small next-token policy (embedding, one hidden layer, output layer) in the packed rows of
x[M, ld]; a tensor of a worker is a view of its row.  In a local step a worker samples tokens from its policy, is
rewarded where the token is the right one for its context, and takes a few optimiser steps on that batch:

    embedding lookup (scaled) -> hidden layer -> logits            dppf_embedding, matrix products
    clipped policy loss, KL term to the first policy, gradient     dppf_policy_loss (the gradient replaces the logits)
    gradients of the layers and of the embedding                   matrix products, dppf_embedding_grad
    one AdamW step over all tensors, states in 8 bits              dppf_adamw_tensors (gradient clipped by its norm)

After `--local-steps` of them the replicas meet in a pull-push round (dppf_consensus).

    python examples/policy_rounds.py --workers 4 --rounds 30
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2507_20424_b200 import binding  # noqa: E402

VOCAB, WIDTH = 100, 40
SHAPES = {"embedding": (VOCAB, WIDTH), "hidden": (WIDTH, WIDTH), "bias": (WIDTH,), "output": (WIDTH, VOCAB)}
SIZES = [math.prod(s) for s in SHAPES.values()]


def views(row):
    """The tensors of one worker in its packed row."""
    return {k: t.view(s) for (k, s), t in zip(SHAPES.items(), row[:sum(SIZES)].split(SIZES))}


def clip_scale(norm):
    """What gradients of this norm are multiplied by, as one CUDA number: a norm that is not finite goes on as it is, so that the
    step is skipped (1 / inf would be 0, and the step a decay of everything, or NaN for an infinite gradient)."""
    return torch.where(torch.isfinite(norm), 1.0 / norm.clamp(min=1.0), norm).view(1)


class Worker:
    def __init__(self, row, grad_row, tokens, scale):
        self.p, self.g, self.tokens, self.scale = views(row), views(grad_row), tokens, scale
        self.optimiser = binding.AdamWTensors([t.view(-1) for t in self.p.values()], [t.view(-1) for t in self.g.values()], state_bits=8,
                                              decay=[0.0 if k == "bias" else 1.0 for k in SHAPES])
        self.policy_ws, self.embedding_ws = binding.alloc_policy_workspace(tokens), binding.alloc_embedding_workspace(tokens, WIDTH)
        self.steps = 0

    def forward(self, context):
        e = binding.dppf_embedding(self.p["embedding"], context, scale=self.scale)
        h = torch.tanh(e @ self.p["hidden"] + self.p["bias"])
        return e, h, h @ self.p["output"]

    def step(self, context, action, old_logp, ref_logp, advantage, lr):
        weight = torch.full_like(advantage, 1.0 / self.tokens)
        e, h, logits = self.forward(context)
        out = binding.dppf_policy_loss(logits, action, old_logp, advantage, weight, ref_logp=ref_logp, kl_coef=0.01, grad_logits=logits, ws=self.policy_ws)
        torch.mm(h.t(), logits, out=self.g["output"])
        dh = (logits @ self.p["output"].t()) * (1 - h * h)
        torch.mm(e.t(), dh, out=self.g["hidden"])
        torch.sum(dh, 0, out=self.g["bias"])
        binding.dppf_embedding_grad(dh @ self.p["hidden"].t(), context, self.g["embedding"], scale=self.scale, ws=self.embedding_ws)
        norm = torch.stack([t.norm() for t in self.g.values()]).norm()
        self.steps += 1
        binding.dppf_adamw_tensors(self.optimiser, lr, 0.9, 0.99, 1e-8, 0.01, self.steps, grad_scale=clip_scale(norm), seed=self.steps)
        return out


def train(workers=4, rounds=30, local_steps=8, tokens=1024, epochs=2, lr=3e-3, alpha=0.1, lam=0.02, seed=0, report=print):
    """Runs the rounds; returns the mean reward of each round and the replicas' mean distance after the last."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d = sum(SIZES)
    x, g = binding.alloc_rows(workers, d, fill=0.0), binding.alloc_rows(workers, d, fill=0.0)
    first = torch.cat([torch.randn(n, generator=gen, device="cuda") * (0.0 if k == "bias" else 0.1 if k == "embedding" else 1 / math.sqrt(WIDTH))
                       for k, n in zip(SHAPES, SIZES)])
    x[:, :d] = first
    team = [Worker(x[m], g[m], tokens, math.sqrt(WIDTH)) for m in range(workers)]
    reference = Worker(first.clone(), torch.zeros_like(first), tokens, math.sqrt(WIDTH))
    right = torch.randperm(VOCAB, generator=gen, device="cuda")                     # the token that a context asks for
    ws, norms = binding.alloc_workspace(workers, d), torch.zeros(workers, device="cuda")
    rewards = []
    for r in range(rounds):
        total = 0.0
        for w in team:
            for _ in range(local_steps):
                context = torch.randint(0, VOCAB, (tokens,), generator=gen, device="cuda")
                logits = w.forward(context)[2]
                action = torch.multinomial(torch.softmax(logits, 1), 1, generator=gen)[:, 0]
                reward = (action == right[context]).float()
                advantage = (reward - reward.mean()) / (reward.std() + 1e-3)
                zero, one = torch.zeros(tokens, device="cuda"), torch.ones(tokens, device="cuda")
                old = binding.dppf_policy_loss(logits, action, zero, zero, one, ws=w.policy_ws).logp                # log-probabilities alone
                ref = binding.dppf_policy_loss(reference.forward(context)[2], action, zero, zero, one, ws=w.policy_ws).logp
                for _ in range(epochs):
                    w.step(context, action, old, ref, advantage, lr)
                total += float(reward.mean())
        binding.dppf_consensus(x, alpha, lam, norms_out=norms, ws=ws, d=d)
        rewards.append(total / (workers * local_steps))
        report(f"round {r + 1:3d}  reward {rewards[-1]:.3f}  distance {float(norms.mean()):.4f}")
    return rewards, float(norms.mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, kind, default in (("workers", int, 4), ("rounds", int, 30), ("local-steps", int, 8), ("tokens", int, 1024), ("lr", float, 3e-3), ("seed", int, 0)):
        ap.add_argument("--" + name, type=kind, default=default)
    train(**{k: v for k, v in vars(ap.parse_args()).items()})
