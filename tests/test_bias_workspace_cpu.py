"""What PositionBias.backward keeps as workspace.  The wrapper's own code runs on tensors in host memory; the library only gives
sizes, and no operator is called."""
import pytest
import torch

from paper_2206_10581_amd import binding as b


@pytest.fixture
def made(monkeypatch):
    """A PositionBias on the host; `made.capturing` says whether its calls are captured, `made.used` which workspaces they had."""
    def init(self, device):
        self.torch, self.device, self.index, self.lib = torch, device, 0, b.load_library()
        self._stream = lambda index: 0

    def call(self, function, *args):
        made.used.append((self._ws_ptr, self.workspace_bytes))

    class Made:
        capturing = False

    made = Made()
    made.used = []
    monkeypatch.setattr(b._OnDevice, "__init__", init)
    monkeypatch.setattr(b._OnDevice, "_call", call)
    monkeypatch.setattr(b._OnDevice, "_capturing", lambda self: made.capturing, raising=False)
    made.bias = b.PositionBias(torch.zeros(32, 16), torch.zeros(4097, dtype=torch.int32))
    return made


def _held(bias):
    spaces = {s.data_ptr(): s.numel() for s in [bias.workspace, *bias._spaces]}
    return sum(spaces.values())


def _grad(n):
    return torch.empty(n).expand(8, 16, n, n)                 # the same row again and again


def _needed(n):
    rc, nbytes = b.tt_emb_bias_workspace_bytes(b.TTEmbPairs(256, 0, 0, 0, n, n, 8, 16, b.TT_EMB_FP32, 0), 2048)
    assert rc == 0
    return nbytes


def test_rising_lengths_keep_one_workspace(made):
    most = 0
    for n in range(8, 1400, 3):
        made.bias.backward(_grad(n))
        most = max(most, _needed(n))
        assert made.used[-1][1] >= _needed(n) and made.used[-1][0] % 256 == 0
        assert _held(made.bias) <= 1.5 * most + 4096
    assert len(set(made.used)) < 40                           # nor is one made for every length


def test_captured_calls_keep_theirs(made):
    """The one that a capture used, whether it was there before or made by it, stays where it is as long as the object does."""
    captured = []
    for n in range(8, 1000, 50):
        made.bias.backward(_grad(n))
        made.capturing = n % 300 == 8
        for more in (0, 7):
            made.bias.backward(_grad(n + more))
            if made.capturing:
                captured.append(made.used[-1])
        made.capturing = False
    kept = {(s.data_ptr() + 255) & ~255: s.numel() - 256 for s in made.bias._spaces}
    assert len(captured) == 8 and set(captured) == set(kept.items())
    assert len(made.bias._spaces) == len(kept)
