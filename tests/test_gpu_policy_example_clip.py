"""examples/policy_rounds.py: a worker's step whose gradients overflow is skipped whole."""
import importlib.util
import os

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("advantage", [1e25, float("inf")])    # a norm that overflows, gradients that are not finite themselves
def test_step_whose_gradients_overflow_is_skipped(advantage):
    require_gpu()
    spec = importlib.util.spec_from_file_location("policy_rounds", os.path.join(ROOT, "examples", "policy_rounds.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    T, d = 64, sum(example.SIZES)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    row = torch.randn(d, generator=gen, device="cuda") * 0.1
    worker = example.Worker(row, torch.zeros_like(row), T, 1.0)
    context, action = (torch.randint(0, example.VOCAB, (T,), generator=gen, device="cuda") for _ in range(2))
    logp = torch.log_softmax(worker.forward(context)[2], 1).gather(1, action[:, None])[:, 0]
    state = lambda: [row.clone()] + [t.view(torch.uint8).clone() for t in (*worker.optimiser.exp_avgs, *worker.optimiser.exp_avg_sqs)]  # noqa: E731
    one = torch.ones(T, device="cuda")
    start = state()
    worker.step(context, action, logp, logp, one, 1e-2)
    before = state()
    assert not torch.equal(before[0], start[0])
    worker.step(context, action, logp, logp, one * advantage, 1e-2)
    assert all(torch.equal(x, y) for x, y in zip(before, state()))
    worker.step(context, action, logp, logp, one, 1e-2)
    assert torch.isfinite(row).all() and not torch.equal(before[0], row)
