"""Tensors that GradientClip takes, and those that it refuses."""
import pytest

pytestmark = pytest.mark.gpu


def test_outputs_in_another_order_of_single_places():
    import torch
    import paper_2206_10581_amd as tt
    a = torch.randn(64, 30, 1, 1, device="cuda")
    out = torch.empty_like(a).to(memory_format=torch.channels_last)
    assert out.stride() != a.stride()
    tt.GradientClip([a], out=[out]).clip(1e9, scale=2.0)
    assert torch.equal(out, 2 * a)
