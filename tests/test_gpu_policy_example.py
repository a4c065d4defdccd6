"""examples/policy_rounds.py: the operators of a local step together with the consensus round learn the task."""
import importlib.util
import os

import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_workers_learn_between_rounds():
    require_gpu()
    spec = importlib.util.spec_from_file_location("policy_rounds", os.path.join(ROOT, "examples", "policy_rounds.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    rewards, distance = example.train(workers=3, rounds=20, local_steps=6, report=lines.append)
    # chance is 1 in 100 tokens; the replicas stay apart (the push) but near each other (the pull)
    assert rewards[0] < 0.1 and rewards[-1] > 0.5, rewards
    assert 0 < distance < 10 and len(lines) == 20
