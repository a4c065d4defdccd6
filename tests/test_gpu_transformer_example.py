"""examples/transformer_rounds.py: it runs, and the gradients of its local step, all operators together, are those of the same
model in 64 bits.

Tolerance: activations, weights and their gradients pass some thirty roundings to bf16 between a parameter and the loss and back (eight a layer
each way, two layers), each 2^-8 of a value at most and by chance up or down: the 2-norm of a gradient is off by about
sqrt(30) 2^-9 = 1.1 %; 5 % is asked for, of the whole tensor's norm."""
import importlib.util
import os

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    require_gpu()
    spec = importlib.util.spec_from_file_location("transformer_rounds", os.path.join(ROOT, "examples", "transformer_rounds.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def model64(e, p, batch, lengths, frequencies):
    """The loss by torch's own operations in 64 bits, sequence by sequence."""
    norm = lambda x, w, b: (x - x.mean(1, keepdim=True)) / (x.var(1, correction=0, keepdim=True) + 1e-5).sqrt() * w + b  # noqa: E731
    at, total, count = 0, 0.0, 0
    for n in lengths:
        ids, targets = batch.ids[at:at + n], batch.targets[at:at + n]
        at += n
        if n == 0:
            continue
        x = p["embedding"][ids]
        angle = torch.arange(n, device="cuda").double()[:, None] * frequencies
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        turn = lambda z: torch.cat((z[..., :e.DIM // 2] * c - z[..., e.DIM // 2:] * s, z[..., e.DIM // 2:] * c + z[..., :e.DIM // 2] * s), -1)  # noqa: E731,B023
        for layer in range(e.LAYERS):
            rows = (norm(x, p[f"{layer}.norm1.w"], p[f"{layer}.norm1.b"]) @ p[f"{layer}.qkv"]).view(n, -1, e.DIM)
            q, k, v = turn(rows[:, :e.HEADS]), turn(rows[:, e.HEADS:e.HEADS + e.KV_HEADS]), rows[:, e.HEADS + e.KV_HEADS:]
            k, v = (t.repeat_interleave(e.HEADS // e.KV_HEADS, 1) for t in (k, v))
            z = torch.einsum("ihd,jhd->hij", q, k) * e.DIM ** -0.5
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
            x = x + torch.einsum("hij,jhd->ihd", torch.softmax(z, -1), v).reshape(n, -1) @ p[f"{layer}.out"]
            x = x + torch.relu(norm(x, p[f"{layer}.norm2.w"], p[f"{layer}.norm2.b"]) @ p[f"{layer}.up"]) @ p[f"{layer}.down"]
        logp = torch.log_softmax(norm(x, p["norm.w"], p["norm.b"]) @ p["output"], 1)
        there = targets >= 0
        total = total - logp[there].gather(1, targets[there][:, None]).sum()
        count += int(there.sum())
    return total / count


def test_gradients_of_a_local_step(example):
    from paper_2507_20424_b200 import binding
    e, gen = example, torch.Generator(device="cuda")
    gen.manual_seed(5)
    row = e.first_row(gen)
    worker = e.Worker(row, torch.full_like(row, float("nan")))
    lengths = [150, 1, 0, 77, 260, 2]
    batch = e.Batch(lengths, gen)
    loss = worker.gradients(batch)
    p = {k: t.double().requires_grad_() for k, t in e.views(row).items()}
    want = model64(e, p, batch, lengths, binding.rotary_frequencies(e.DIM)[0])
    want.backward()
    want = float(want.detach())
    assert abs(float(loss) - want) < 0.02 * want
    for k, t in p.items():
        off = float((worker.g[k].double() - t.grad).norm() / t.grad.norm())
        assert off < 0.05, (k, off)
    again = e.Worker(row, torch.zeros_like(row))
    again.gradients(batch)
    assert all(torch.equal(worker.g[k], again.g[k]) for k in p)                # the same bits from run to run


def test_rounds_run(example):
    lines = []
    losses, distance = example.train(workers=2, rounds=2, local_steps=2, report=lines.append)
    assert len(losses) == len(lines) == 2 and all(x == x and x < 100 for x in losses) and 0 < distance < 100
