"""The example that takes a training step through all operators together: it learns, with the schemes that send least."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("algo", ["fp16", "efsign", "topk"])
def test_the_example_learns(algo):
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    rewards = module.train(algo, iterations=40)
    # one action in ten pays; the mean of 1024 samples is off by 0.01
    assert abs(rewards[0] - 0.1) < 0.05
    assert rewards[-1] > 0.2, rewards
