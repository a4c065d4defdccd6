"""Workers that train a small transformer on packed sequences between consensus rounds, on one GPU.

M workers hold replicas in the packed rows of x[M, ld], fp32; a tensor of a worker is a view of its row.  Sequences of different
lengths are packed into one batch of tokens, activations are bf16 and the stream that the layers add to is fp32.  A local step:

    embedding lookup                                               dppf_embedding
    each layer:  norm of the stream and what was added to it       dppf_layer_norm (branch)
                 queries, keys, values of one product, turned      dppf_rotary, in place
                 attention within the sequences                    dppf_attention (one plan for the batch and all layers)
                 norm, two products with a rectifier
    norm, logits, loss and its gradient                            dppf_layer_norm, dppf_policy_loss (ratios of one: cross entropy's gradient)
    the same backward                                              dppf_layer_norm_grad, dppf_attention_grad, dppf_rotary (inverse), dppf_embedding_grad
    one AdamW step over all tensors                                dppf_adamw_tensors

After `--local-steps` of them the replicas meet in a pull-push round (dppf_consensus).  The task: name the token before the last one.

    python examples/transformer_rounds.py --workers 2 --rounds 20
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2507_20424_b200 import binding  # noqa: E402

VOCAB, WIDTH, HEADS, KV_HEADS, DIM, INNER, LAYERS = 64, 128, 4, 2, 32, 256, 2
BF16 = torch.bfloat16


def shapes():
    s = {"embedding": (VOCAB, WIDTH), "norm.w": (WIDTH,), "norm.b": (WIDTH,), "output": (WIDTH, VOCAB)}
    for n in range(LAYERS):
        s |= {f"{n}.norm1.w": (WIDTH,), f"{n}.norm1.b": (WIDTH,), f"{n}.qkv": (WIDTH, (HEADS + 2 * KV_HEADS) * DIM), f"{n}.out": (HEADS * DIM, WIDTH),
              f"{n}.norm2.w": (WIDTH,), f"{n}.norm2.b": (WIDTH,), f"{n}.up": (WIDTH, INNER), f"{n}.down": (INNER, WIDTH)}
    return s


SHAPES = shapes()
SIZES = [math.prod(s) for s in SHAPES.values()]


def views(row):
    """The tensors of one worker in its packed row."""
    return {k: t.view(s) for (k, s), t in zip(SHAPES.items(), row[:sum(SIZES)].split(SIZES))}


def first_row(generator):
    """Values to start from: norms at one and zero, the others small."""
    parts = []
    for k, s in SHAPES.items():
        noise = torch.randn(math.prod(s), generator=generator, device="cuda")
        parts.append(torch.ones_like(noise) if k.endswith("norm.w") or k.endswith(("norm1.w", "norm2.w")) else torch.zeros_like(noise) if len(s) == 1
                     else noise * (0.5 if k == "embedding" else 1 / math.sqrt(s[0])))
    return torch.cat(parts)


class Batch:
    """Packed sequences: tokens, positions within their sequence, and the plan."""

    def __init__(self, lengths, generator):
        self.tokens = sum(lengths)
        starts = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32)
        self.positions = torch.cat([torch.arange(n) for n in lengths]).cuda()
        self.plan = binding.AttentionPlan(starts.cuda(), self.tokens)
        self.ids = torch.randint(0, VOCAB, (self.tokens,), generator=generator, device="cuda")
        before = torch.cat([self.ids.new_zeros(1), self.ids[:-1]])
        self.targets = torch.where(self.positions > 0, before, -100)       # a sequence's first token has none


class Worker:
    def __init__(self, row, grad_row):
        self.p, self.g = views(row), views(grad_row)
        self.frequencies, self.scale = binding.rotary_frequencies(DIM)
        self.optimiser = binding.AdamWTensors([t.view(-1) for t in self.p.values()], [t.view(-1) for t in self.g.values()], state_bits=8,
                                              decay=[1.0 if t.dim() > 1 else 0.0 for t in self.p.values()])
        self.steps = 0

    def forward(self, batch):
        """Logits, and what the way back needs."""
        p, kept = self.p, []
        w = {k: t.to(BF16) for k, t in p.items() if t.dim() > 1 and k != "embedding"}
        stream, branch = binding.dppf_embedding(p["embedding"], batch.ids), None
        for n in range(LAYERS):
            n1 = binding.dppf_layer_norm(stream, p[f"{n}.norm1.w"], p[f"{n}.norm1.b"], branch=branch, out_dtype=BF16)
            rows = (n1.out @ w[f"{n}.qkv"]).view(batch.tokens, HEADS + 2 * KV_HEADS, DIM)
            turned = rows[:, :HEADS + KV_HEADS]
            binding.dppf_rotary(turned, batch.positions, self.frequencies, scale=self.scale, out=turned)
            a = binding.dppf_attention(rows[:, :HEADS], rows[:, HEADS:HEADS + KV_HEADS], rows[:, HEADS + KV_HEADS:], batch.plan)
            n2 = binding.dppf_layer_norm(n1.sum, p[f"{n}.norm2.w"], p[f"{n}.norm2.b"], branch=a.out.view(batch.tokens, -1) @ w[f"{n}.out"], out_dtype=BF16)
            up = torch.relu(n2.out @ w[f"{n}.up"])
            stream, branch = n2.sum, up @ w[f"{n}.down"]
            kept.append((n1, rows, a, n2, up))
        last = binding.dppf_layer_norm(stream, p["norm.w"], p["norm.b"], branch=branch, out_dtype=BF16)
        return last.out @ w["output"], (w, kept, last)

    def gradients(self, batch):
        """Fills the gradients of the mean of -log probability of the targets; returns the loss."""
        logits, (w, kept, last) = self.forward(batch)
        there = batch.targets >= 0
        weight = there.float() / there.sum()
        one = torch.ones_like(weight)
        # an advantage of one and a ratio of one: the loss's gradient is that of -log probability
        logp = binding.dppf_policy_loss(logits, batch.targets, torch.zeros_like(one), one, weight).logp
        binding.dppf_policy_loss(logits, batch.targets, logp, one, weight, grad_logits=logits)
        g = self.g
        g["output"].copy_(last.out.t() @ logits)
        stream = binding.dppf_layer_norm_grad(logits @ w["output"].t(), last.sum, last.mean, last.rstd, self.p["norm.w"], g["norm.w"], g["norm.b"])
        for n in reversed(range(LAYERS)):
            n1, rows, a, n2, up = kept[n]
            branch = stream.to(BF16)
            g[f"{n}.down"].copy_(up.t() @ branch)
            d_up = (branch @ w[f"{n}.down"].t()) * (up > 0)
            g[f"{n}.up"].copy_(n2.out.t() @ d_up)
            stream = binding.dppf_layer_norm_grad(d_up @ w[f"{n}.up"].t(), n2.sum, n2.mean, n2.rstd, self.p[f"{n}.norm2.w"], g[f"{n}.norm2.w"], g[f"{n}.norm2.b"], grad_sum=stream, grad_x=stream)
            branch = stream.to(BF16)
            g[f"{n}.out"].copy_(a.out.view(batch.tokens, -1).t() @ branch)
            d_rows = torch.empty_like(rows)
            cut = (slice(0, HEADS), slice(HEADS, HEADS + KV_HEADS), slice(HEADS + KV_HEADS, None))
            q, k, v = (rows[:, c] for c in cut)
            binding.dppf_attention_grad((branch @ w[f"{n}.out"].t()).view(batch.tokens, HEADS, DIM), q, k, v, a.out, a.lse, batch.plan,
                                        grad_q=d_rows[:, cut[0]], grad_k=d_rows[:, cut[1]], grad_v=d_rows[:, cut[2]])
            turned = d_rows[:, :HEADS + KV_HEADS]
            binding.dppf_rotary(turned, batch.positions, self.frequencies, scale=self.scale, inverse=True, out=turned)
            d_rows = d_rows.view(batch.tokens, -1)
            g[f"{n}.qkv"].copy_(n1.out.t() @ d_rows)
            stream = binding.dppf_layer_norm_grad(d_rows @ w[f"{n}.qkv"].t(), n1.sum, n1.mean, n1.rstd, self.p[f"{n}.norm1.w"], g[f"{n}.norm1.w"], g[f"{n}.norm1.b"], grad_sum=stream, grad_x=stream)
        binding.dppf_embedding_grad(stream, batch.ids, g["embedding"])
        return -(logp * weight).sum()

    def step(self, batch, lr):
        loss = self.gradients(batch)
        self.steps += 1
        binding.dppf_adamw_tensors(self.optimiser, lr, 0.9, 0.99, 1e-8, 0.01, self.steps, seed=self.steps)
        return loss


def train(workers=2, rounds=20, local_steps=8, lr=3e-3, alpha=0.1, lam=0.02, seed=0, report=print):
    """Runs the rounds; returns the mean loss of each round and the replicas' mean distance after the last."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d = sum(SIZES)
    x, g = binding.alloc_rows(workers, d, fill=0.0), binding.alloc_rows(workers, d, fill=0.0)
    x[:, :d] = first_row(gen)
    team = [Worker(x[m], g[m]) for m in range(workers)]
    ws, norms = binding.alloc_workspace(workers, d), torch.zeros(workers, device="cuda")
    losses = []
    for r in range(rounds):
        total = 0.0
        for w in team:
            for _ in range(local_steps):
                total += float(w.step(Batch([200, 1, 57, 130, 0, 300], gen), lr))
        binding.dppf_consensus(x, alpha, lam, norms_out=norms, ws=ws, d=d)
        losses.append(total / (workers * local_steps))
        report(f"round {r + 1:3d}  loss {losses[-1]:.3f}  distance {float(norms.mean()):.4f}")
    return losses, float(norms.mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, kind, default in (("workers", int, 2), ("rounds", int, 20), ("local-steps", int, 8), ("lr", float, 3e-3), ("seed", int, 0)):
        ap.add_argument("--" + name, type=kind, default=default)
    train(**{k: v for k, v in vars(ap.parse_args()).items()})
