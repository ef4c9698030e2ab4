"""The example's gradients cover all that its steps look up."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_row_that_was_looked_up_has_its_gradient(monkeypatch):
    import torch
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "train_nodes_and_tokens.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    seen = {"looked up": 0, "updated": 0, "clipped": [], "applied": []}

    class Nodes(example.TTEmbedding):
        def forward(self, ids, out=None):
            seen["looked up"] += ids.numel()
            return super().forward(ids, out)

        def forward_eval(self, ids, out=None):
            seen["looked up"] += ids.numel()
            return super().forward_eval(ids, out)

        def backward_update(self, grad_out, lr):
            assert bool(grad_out.any(1).all())          # no row without a gradient
            seen["updated"] += grad_out.shape[0]
            seen["applied"].append(grad_out.double().square().sum().item())
            return super().backward_update(grad_out, lr)

    class Clip(example.GradientClip):
        def clip(self, max_norm, **more):
            seen["clipped"].append([t.double().square().sum().item() for t in self.tensors])
            return super().clip(max_norm, **more)

    monkeypatch.setattr(example, "TTEmbedding", Nodes)
    monkeypatch.setattr(example, "GradientClip", Clip)
    _, norms = example.train(steps=5)
    assert seen["looked up"] == seen["updated"] == 5 * example.BATCH * example.MICRO
    for norm, parts, applied in zip(norms, seen["clipped"], seen["applied"]):
        assert abs(norm - sum(parts) ** 0.5) <= norm * 2.0 ** -22
        factor = min(1.0, 0.5 / (norm + 1e-6))
        assert abs(applied - parts[2] * factor ** 2) <= applied * 1e-6
