"""Which table DenseEmbedding hands to the library when its weight changes between calls.  The wrapper's own code runs on
tensors in host memory; its calls of the library are recorded and none is made."""
import pytest
import torch

from paper_2206_10581_amd import binding as b


@pytest.fixture
def made(monkeypatch):
    """Makes DenseEmbeddings on the host; their calls are left in `made.calls` as (function, matrices)."""
    def init(self, device):
        self.torch, self.device, self.index, self.lib = torch, device, 0, b.load_library()
        self._stream = lambda index: 0
        self._home = 0

    def call(self, function, *args):
        made.calls.append((function.__name__, [a._obj for a in args if hasattr(a, "_obj")]))

    def made(weight, max_batch=8, **more):
        return b.DenseEmbedding(weight, max_batch, **more)

    made.calls = []
    monkeypatch.setattr(b._OnDevice, "__init__", init)
    monkeypatch.setattr(b._OnDevice, "_call", call)
    return made


KINDS = {torch.float32: b.TT_EMB_FP32, torch.bfloat16: b.TT_EMB_BF16, torch.float16: b.TT_EMB_FP16}


def _is(m, t):
    return (m.data, m.rows, m.cols, m.type) == (t.data_ptr(), t.shape[0], t.shape[1], KINDS[t.dtype]) and \
        m.ld == (t.stride(0) if t.shape[0] > 1 else t.shape[1])


CHANGES = {
    "every second row": lambda w: w[::2],
    "fewer rows": lambda w: w[:4],
    "one row": lambda w: w[:1],
    "narrower": lambda w: w[:, :8],
    "of half the bytes": lambda w: w.view(torch.bfloat16),
    "another type of the same size": lambda w: w[:, :8].view(torch.bfloat16).view(torch.float16),
    "rows put together": lambda w: w.view(6, 32),
    "another place": lambda w: w[1:],
    "grown": lambda w: torch.zeros(40, 16),
    "grown and wider": lambda w: torch.zeros(40, 700),
}


@pytest.mark.parametrize("change", CHANGES.values(), ids=CHANGES.keys())
def test_the_table_is_the_weight_of_the_call(made, change):
    weight = torch.nn.Parameter(torch.zeros(12, 16), requires_grad=False)
    emb = made(weight)
    emb.forward(torch.zeros(3, dtype=torch.int64))
    weight.data = change(weight.data)
    rows, dim = weight.shape
    assert (emb.rows, emb.dim) == (rows, dim)
    ids = torch.zeros(3, dtype=torch.int64)
    made.calls.clear()
    out = emb.forward(ids)
    assert out.shape == (3, dim) and out.dtype == weight.dtype and _is(made.calls[0][1][0], weight)
    grad = torch.zeros(3, dim)
    assert emb.backward(ids, grad).shape == (rows, dim)
    into = torch.zeros(rows, dim)
    assert emb.backward(ids, grad, out=into) is into and _is(made.calls[-1][1][1], into)
    emb.backward_update(ids, grad, 0.5)
    assert made.calls[-1][0] == "tt_emb_dense_backward" and _is(made.calls[-1][1][1], weight)
    # the workspace is large enough for the width of the call
    assert emb.workspace_bytes >= b.tt_emb_dense_workspace_bytes(dim, 8)[1]
    assert emb._ws_ptr + emb.workspace_bytes <= emb.workspace.data_ptr() + emb.workspace.numel()
    with pytest.raises(ValueError):
        emb.backward(ids, torch.zeros(3, dim + 1))
    with pytest.raises(ValueError):
        emb.backward(ids, grad, out=torch.zeros(rows + 1, dim))


@pytest.mark.parametrize("change", [lambda w: w.t(), lambda w: w[0], lambda w: w[:, :0], lambda w: w.double(),
                                    lambda w: w[:, ::2], lambda w: w[:1].expand(5, 16)])
def test_a_weight_that_is_no_table_any_more_is_refused(made, change):
    weight = torch.nn.Parameter(torch.zeros(12, 16), requires_grad=False)
    emb = made(weight)
    weight.data = change(weight.data)
    for _ in range(2):
        with pytest.raises(ValueError):
            emb.forward(torch.zeros(3, dtype=torch.int64))
        with pytest.raises(ValueError):
            emb.backward_update(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 16), 1.0)
    assert not made.calls


def test_a_weight_that_stays_is_described_once(made):
    weight = torch.zeros(12, 16)
    emb = made(weight)
    table, space = emb._table, emb.workspace
    emb.forward(torch.zeros(3, dtype=torch.int64))
    emb.backward_update(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 16), 1.0)
    assert emb._table is table and emb.workspace is space


def test_a_workspace_stays_when_a_larger_one_takes_its_place(made):
    """A captured graph holds its address."""
    weight = torch.nn.Parameter(torch.zeros(12, 16), requires_grad=False)
    emb = made(weight)
    import weakref
    first, at = weakref.ref(emb.workspace), emb._ws_ptr
    weight.data = torch.zeros(12, 700)
    emb.forward(torch.zeros(3, dtype=torch.int64))
    assert emb._ws_ptr != at and first() is not None
