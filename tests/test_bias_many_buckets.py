"""A table of 2^31 - 1 buckets, the most that there may be: every row of its gradient is written, and nothing before it."""
import pytest

pytestmark = pytest.mark.gpu


def test_the_largest_table():
    import torch
    import paper_2206_10581_amd as tt
    n = (1 << 31) - 1
    named = [0, n - (1 << 20) - 1, n - (1 << 20), n - 1]       # a grid of 2^20 blocks takes the last ones in its last step
    room = torch.full((n + 64, 1), 5.0, dtype=torch.bfloat16, device="cuda")
    table = room[64:]
    of = torch.tensor([named[0], named[1], named[2], named[3], -1], dtype=torch.int32, device="cuda")
    bias = tt.PositionBias(table, of)
    grad = torch.tensor([1.0, 2.0, 3.0, 4.0, 6.0], device="cuda").view(1, 1, 1, 5)
    assert bias.backward(grad, -2, out=table) is table
    assert [table[u].item() for u in named] == [1.0, 2.0, 3.0, 4.0]
    assert sum(int(torch.count_nonzero(part)) for part in table.split(1 << 28)) == 4
    assert bool((room[:64] == 5.0).all())
    # and as a table
    assert bias.forward(1, 5, -2).flatten().tolist() == [1.0, 2.0, 3.0, 4.0, 0.0]
