"""The fine-tuning example: losses, their gradients, clipping and both optimizers as one training step."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_learns():
    """The preference loss starts at log 2 (the model is its own reference) and falls, and the sampled
    answers follow the rule more often after the policy phase than before it."""
    import __graft_entry__

    __graft_entry__.build()
    spec = importlib.util.spec_from_file_location("finetune", os.path.join(ROOT, "examples", "finetune.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, rewards = example.main(steps=60)
    assert abs(losses[0] - math.log(2)) < 1e-3, losses  # bf16 logits of two equal models are equal: the margin is 0
    assert losses[-1] < 0.5 * losses[0], losses
    assert all(math.isfinite(x) for x in losses) and rewards[-1] > rewards[0] and rewards[-1] > 0.5, rewards
