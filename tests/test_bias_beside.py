"""Biases added beside the scores in one buffer, and over them; what else shares memory with the scores is refused."""
import pytest

pytestmark = pytest.mark.gpu


def _made():
    import torch
    import paper_2206_10581_amd as tt
    of = tt.PositionBias.log_buckets(8, 20)
    return tt.PositionBias(torch.randn((8, 3), generator=torch.Generator().manual_seed(1)).cuda(), of.cuda())


def _room(*shape):
    import torch
    return torch.randn(shape, generator=torch.Generator().manual_seed(2)).cuda()


def test_beside_each_other_in_one_buffer():
    import torch
    bias = _made()
    batch, heads, queries, keys = 2, 3, 9, 50
    layouts = [(_room(2, batch, heads, queries, keys), lambda r: (r[0], r[1])),
               (_room(batch, heads, queries, 2 * keys), lambda r: (r[..., :keys], r[..., keys:])),
               (_room(batch, heads, 2 * queries, keys), lambda r: (r[:, :, 1::2], r[:, :, ::2])),
               (_room(batch, 2, heads, queries, keys), lambda r: (r[:, 1], r[:, 0])),
               (_room(batch, queries, 2, heads, keys + 3), lambda r: (r[:, :, 0, :, 1:-2].transpose(1, 2), r[:, :, 1, :, 3:].transpose(1, 2))),
               (_room(4, heads, queries, keys), lambda r: (r[:1].expand(3, -1, -1, -1), r[1:]))]
    for room, cut in layouts:
        before = room.clone()
        scores, out = cut(room)
        given, _ = cut(before)
        want = bias.add_to(given, -4, out=torch.empty(out.shape, device="cuda"))
        assert bias.add_to(scores, -4, out=out) is out and torch.equal(out, want)
        assert torch.equal(scores, given)
        where = torch.zeros_like(room, dtype=torch.bool)      # nothing else was written
        cut(where)[1].fill_(True)
        assert torch.equal(room[~where], before[~where])


def test_beside_each_other_in_two_types():
    """Scores in fp32 and an output in bf16, in rows of one buffer, on either side."""
    import torch
    import paper_2206_10581_amd as tt
    bias = _made()
    room = _room(2, 3, 9, 90)
    for scores, out in ((room[..., :50], room.view(torch.bfloat16)[..., 100:150]),
                        (room[..., 25:75], room.view(torch.bfloat16)[..., :50])):
        given = scores.clone()
        want = bias.add_to(given, -4, out=torch.empty(out.shape, dtype=torch.bfloat16, device="cuda"))
        assert torch.equal(bias.add_to(scores, -4, out=out), want) and torch.equal(scores, given)
    for first in (99, 49):                                     # a place too early
        with pytest.raises(tt.TTEmbError):
            bias.add_to(room[..., :50], out=room.view(torch.bfloat16)[..., first:first + 50])


def test_over_the_scores():
    import torch
    bias, x = _made(), _room(2, 3, 9, 50)
    want = bias.add_to(x, out=torch.empty_like(x))
    for out in (None, x.view(2, 3, 9, 50), x.unsqueeze(0)[0]):
        y = x.clone()
        assert torch.equal(bias.add_to(y, out=None if out is None else y.view(2, 3, 9, 50)), want) and torch.equal(y, want)


def test_anything_between_is_refused():
    import torch
    import paper_2206_10581_amd as tt
    bias, room = _made(), _room(3, 3, 9, 51)
    half = torch.zeros((2, 3, 9, 50), dtype=torch.bfloat16, device="cuda")
    before = room.clone()
    for scores, out in ((room[..., :50], room[..., 1:]), (room[:2], room[1:]), (room[:, :, :8], room[:, :, 1:]),
                        (half, half.view(torch.float16)), (room[:1].expand(3, -1, -1, -1), room),
                        (room.view(-1)[:1350].view(1, 3, 9, 50), room.view(-1)[7:1357].view(1, 9, 3, 50).transpose(1, 2))):
        with pytest.raises(tt.TTEmbError):
            bias.add_to(scores, out=out)
    assert torch.equal(room, before) and bool((half == 0).all())
