"""The example that trains a tensor-train table and a plain one together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_lowers_the_loss():
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "train_nodes_and_tokens.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms = example.train(steps=80)
    assert max(norms) > 0.5          # some steps are clipped
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0], losses
    assert example.train(steps=80)[0] == losses      # every sum has a fixed order
