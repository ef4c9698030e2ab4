"""A plain table whose memory, shape, strides or type change between calls, its address among what may stay the same."""
import pytest

pytestmark = pytest.mark.gpu

CHANGES = {
    "every second row": lambda w: w[::2],
    "fewer rows": lambda w: w[:7],
    "narrower": lambda w: w[:, :24],
    "of half the bytes": lambda w: w.view(w.new_empty(0).bfloat16().dtype),
    "rows put together": lambda w: w.view(20, 120),
    "grown": lambda w: w.repeat(3, 1),
    "grown and wider": lambda w: w.repeat(3, 20),
}


@pytest.mark.parametrize("B", [30, 1500])
@pytest.mark.parametrize("change", CHANGES.values(), ids=CHANGES.keys())
def test_calls_take_the_weight_as_it_is(change, B):
    """Whole numbers, so that every sum is exact in fp32 and in bf16."""
    import torch
    import paper_2206_10581_amd as tt
    g = torch.Generator().manual_seed(B)
    flat = torch.full((4000,), 3.0, device="cuda")     # the table's memory and what lies behind it
    flat[:2400] = torch.randint(-8, 9, (2400,), generator=g).float().cuda()
    weight = torch.nn.Parameter(flat[:2400].view(40, 60), requires_grad=False)
    emb = tt.DenseEmbedding(weight, B, scale=2.0)
    emb.forward(torch.zeros(1, dtype=torch.int64, device="cuda"))
    weight.data = change(weight.data)
    rows, dim = weight.shape
    ids = torch.randint(-3, rows + 60, (B,), generator=g).cuda()
    inside = (ids >= 0) & (ids < rows)
    before = flat.clone()
    got = emb.forward(ids, dtype=torch.float32)
    want = torch.where(inside[:, None], weight[torch.where(inside, ids, 0)].float() * 2, 0.0)
    assert got.shape == (B, dim) and torch.equal(got, want)
    grad = (torch.arange(B, device="cuda")[:, None] % 3 - 1 + torch.arange(dim, device="cuda") % 2).float()
    sums = torch.zeros(rows, dim, device="cuda").index_add_(0, ids[inside], grad[inside])
    assert torch.equal(emb.backward(ids, grad, dtype=torch.float32), 2 * sums)
    old = weight.data.double().clone()
    emb.backward_update(ids, grad, 0.25)
    want = (old - 0.5 * sums.double()).to(weight.dtype)
    assert torch.equal(weight.data, want)
    assert torch.equal(flat[2400:], before[2400:])     # nothing behind the table is written
