"""Position bias by buckets and its gradient, against plain forms in 64 bits.

Tolerances.  u = 2^-24.  A bias alone is rounded once, to the output's type; added to a score it is one sum in fp32 (u) and that
rounding.  The gradient's sums: a part of at least 16 rows is summed in fp32, the rest in fp64.  A lane meets every 64th
piece of every fourth group of four rows, so it adds up to 4 (keys / 64 + 8) values for a group of rows, one after the other where
some of a piece count and others do not; of short rows a thread adds the min(queries, keys) values of a diagonal; then come
6 + 4 joins and the sum of a thread's diagonals, of which there are (queries + keys) / 256.  A part of all rows of a sequence
would thus need 24 + (queries / 16 + 1) * 4 (keys / 64 + 8) + (queries + keys) / 256 additions at most, and one of all sequences that times
their number.  That bound tells little of a value that is missing or taken twice, so whole numbers, whose sums are exact, are
compared too."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TYPES = ["float32", "bfloat16", "float16"]


def _normal(seed, shape, kind):
    import torch
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(getattr(torch, kind)).cuda()


def _map(how):
    """Bucket maps: (bucket_of, buckets)."""
    import torch
    import paper_2206_10581_amd as tt
    if how == "both":
        return tt.PositionBias.log_buckets(32, 128), 32
    if how == "causal":
        return tt.PositionBias.log_buckets(16, 50, bidirectional=False), 16
    if how == "far":
        return tt.PositionBias.log_buckets(32, 5000), 32
    if how == "each":
        return torch.arange(401, dtype=torch.int32), 401
    if how == "wide":                         # a bucket for each of 3001 distances
        return torch.arange(3001, dtype=torch.int32), 3001
    if how == "one":
        return torch.zeros(1, dtype=torch.int32), 1
    if how == "mixed":                        # no order, holes, buckets that nothing names, numbers outside the table
        return torch.from_numpy(np.random.default_rng(5).integers(-3, 12, 141).astype(np.int32)), 10
    if how == "none":
        return torch.full((7,), -1, dtype=torch.int32), 3
    raise ValueError(how)


def _buckets(of, offset, batch, queries, keys):
    """[batch, queries, keys], in whole numbers of any size."""
    span = len(of) // 2
    of = of.tolist()
    offsets = offset.tolist() if hasattr(offset, "tolist") else [offset] * batch
    rows = []
    for o in offsets:
        line = [of[min(max(d + o, -span), span) + span] for d in range(1 - queries, keys)]
        line = np.array(line)
        rows.append(np.stack([line[queries - 1 - i:queries - 1 - i + keys] for i in range(queries)]))
    return np.stack(rows)


MAPS = ["both", "causal", "far", "each", "one", "mixed", "none"]
# batch, heads, queries, keys
SIZES = [(1, 1, 1, 1), (3, 2, 1, 300), (2, 3, 40, 1), (2, 3, 17, 33), (1, 2, 129, 515), (2, 1, 300, 1100), (5, 2, 64, 64), (1, 3, 7, 2051),
         (1, 2, 70, 1024), (1, 1, 40, 2000)]


# many heads, so that a part holds several sequences; short rows; many buckets
MORE = [("both", (20, 300, 7, 40)), ("each", (9, 70, 33, 100)), ("both", (2, 3, 2000, 5)), ("causal", (3, 2, 2500, 64)),
        ("wide", (2, 5, 300, 1100)), ("wide", (2, 3, 700, 20)), ("far", (3, 300, 9, 300))]


def _offsets(kind, batch, queries, keys):
    import torch
    if kind == "number":
        return queries - keys
    rng = np.random.default_rng(batch + queries)
    some = [0, 1 - keys, queries, -(1 << 62), (1 << 62), 4_000_000_000, -130]
    return torch.tensor([some[k % len(some)] if kind == "far" else int(rng.integers(-keys, queries + 1)) for k in range(batch)],
                        device="cuda")


def _check(got, ref, tol, kind):
    import torch
    got = got.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        off = np.abs(got - ref) - (tol + U[kind] * np.abs(ref) + 2.0 ** -24 * (kind == "float16"))
    off = np.where((got == ref) | (np.isnan(got) & np.isnan(ref)), -1.0, off)
    assert off.size == 0 or (off <= 0).all(), np.nanmax(off)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("how", MAPS)
def test_bias(how, size):
    import torch
    import paper_2206_10581_amd as tt
    batch, heads, queries, keys = size
    of, n = _map(how)
    for kind, out_kind, offsets, fill in (("float32", "float32", "number", 0.0), ("bfloat16", "float16", "ragged", -math.inf),
                                          ("float16", "bfloat16", "far", 1.5)):
        table = _normal(1, (n, heads + 1), kind)[:, :heads]
        bias = tt.PositionBias(table, of.cuda(), fill)
        offset = _offsets(offsets, batch, queries, keys)
        buckets = _buckets(of, offset, batch, queries, keys)
        padded = np.concatenate([table.double().cpu().numpy(), np.full((1, heads), fill)])
        ref = padded[np.where((buckets >= 0) & (buckets < n), buckets, n)].transpose(0, 3, 1, 2)
        got = bias.forward(queries, keys, offset, dtype=getattr(torch, out_kind))
        assert got.shape == (batch if offsets != "number" else 1, heads, queries, keys)
        _check(got, ref[:got.shape[0]], 0.0, out_kind)
        # into a larger buffer: other places keep what they hold; queries before heads in memory
        room = torch.full((batch, queries + 1, heads, keys + 3), 9.0, dtype=getattr(torch, out_kind), device="cuda")
        view = room[:, :queries, :, 1:keys + 1].transpose(1, 2)
        assert bias.forward(queries, keys, offset, out=view) is view
        _check(view, ref, 0.0, out_kind)
        assert bool((room[:, queries] == 9.0).all()) and bool((room[..., 0] == 9.0).all()) and bool((room[..., keys + 1:] == 9.0).all())
        # added, to another buffer, and in place
        scores = _normal(2, (batch, heads, queries, keys + 1), kind)[..., 1:]
        total = scores.double().cpu().numpy() + ref
        _check(bias.add_to(scores, offset, out=view), total, u * np.abs(np.where(np.isfinite(total), total, 0)), out_kind)
        want = bias.add_to(scores, offset, out=torch.empty(scores.shape, dtype=scores.dtype, device="cuda"))
        assert bias.add_to(scores, offset) is scores and torch.equal(scores, want)


def _sums(grad, buckets, n):
    """Sums and sums of magnitudes by bucket, in 64 bits."""
    g = grad.double().cpu().numpy()
    total, size = np.zeros((n, g.shape[1])), np.zeros((n, g.shape[1]))
    keep = (buckets >= 0) & (buckets < n)
    g = g.transpose(0, 2, 3, 1)
    np.add.at(total, buckets[keep], g[keep])
    np.add.at(size, buckets[keep], np.abs(g[keep]))
    return total, size


def _roundings(batch, queries, keys):
    return batch * (24 + (queries / 16 + 1) * 4 * (keys / 64 + 8) + min(queries, keys) + (queries + keys) / 256)


@pytest.mark.parametrize("how,size", [(how, size) for how in MAPS for size in SIZES] + MORE)
def test_gradient(how, size):
    import torch
    import paper_2206_10581_amd as tt
    batch, heads, queries, keys = size
    of, n = _map(how)
    for kind, out_kind, offsets in (("float32", "float32", "number"), ("bfloat16", "float32", "ragged"),
                                    ("float16", "bfloat16", "far"), ("bfloat16", "float16", "number")):
        table = torch.zeros((n, heads + 2), dtype=getattr(torch, out_kind), device="cuda")[:, 1:heads + 1]
        bias = tt.PositionBias(table, of.cuda())
        offset = _offsets(offsets, batch, queries, keys)
        buckets = _buckets(of, offset, batch, queries, keys)
        # queries before heads in memory, unused keys around
        grad = _normal(3, (batch, queries, heads, keys + 3), kind)[..., 2:keys + 2].transpose(1, 2)
        total, size_of = _sums(grad, buckets, n)
        bound = _roundings(batch, queries, keys) * u * size_of
        got = bias.backward(grad, offset)
        _check(got, total, bound, out_kind)
        assert torch.equal(got, bias.backward(grad, offset))
        room = torch.full((n, heads + 1), 2.0, dtype=getattr(torch, out_kind), device="cuda")
        bias.backward(grad, offset, out=room[:, :heads], add=True)
        _check(room[:, :heads], total + 2.0, bound + u * (np.abs(total) + 2), out_kind)
        assert bool((room[:, heads] == 2.0).all())


@pytest.mark.parametrize("how,size", [(how, size) for how in MAPS for size in SIZES] + MORE)
def test_gradient_of_whole_numbers(how, size):
    """Numbers from -4 to 4, whose sums stay below 2^24: exact in any order."""
    import torch
    import paper_2206_10581_amd as tt
    batch, heads, queries, keys = size
    of, n = _map(how)
    for kind, offsets, gap in (("float32", "number", 0), ("bfloat16", "ragged", 1), ("float16", "far", 8), ("bfloat16", "number", 0)):
        bias = tt.PositionBias(torch.zeros((n, heads), device="cuda"), of.cuda())
        offset = _offsets(offsets, batch, queries, keys)
        g = torch.Generator().manual_seed(7)
        grad = torch.randint(-4, 5, (batch, heads, queries, keys + gap), generator=g).to(getattr(torch, kind)).cuda()[..., :keys]
        total, size_of = _sums(grad, _buckets(of, offset, batch, queries, keys), n)
        assert size_of.max() < 2 ** 24
        assert np.array_equal(bias.backward(grad, offset).double().cpu().numpy(), total)


def test_gradient_of_a_broadcast_and_against_differences():
    """An expanded gradient (one for all sequences), and the slope of sum(grad * bias) in each value of the table, which is linear."""
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    table = _normal(1, (n, 3), "float32")
    bias = tt.PositionBias(table, of.cuda())
    one = _normal(2, (1, 3, 50, 200), "float32")
    grad = one.expand(4, 3, 50, 200)
    got = bias.backward(grad, -150)
    total, size = _sums(grad, _buckets(of, -150, 4, 50, 200), n)
    _check(got, total, _roundings(4, 50, 200) * u * size, "float32")
    for row in (0, 5, 15, 16, 31):
        up = table.clone()
        up[row] += 1.0
        there, here = (tt.PositionBias(t, of.cuda()).forward(50, 200, -150).double() for t in (up, table))
        slope = 4 * (one.double() * (there - here))[0].sum((1, 2))
        # table values below 4: each difference of biases is off by 2 * 4 u
        assert (slope - got[row].double()).abs().max() <= size[row].max() * (_roundings(4, 50, 200) + 16) * u


def test_masked_places():
    """NaN and infinities where there is no bucket reach nothing; an infinite bias replaces the score."""
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("causal")
    table = _normal(1, (n, 2), "float32")
    table[3, 0] = -math.inf
    bias = tt.PositionBias(table, of.cuda(), fill=-math.inf)
    buckets = _buckets(of, 0, 2, 40, 90)
    grad = _normal(2, (2, 2, 40, 90), "bfloat16")
    want = bias.backward(grad, 0, dtype=torch.float32)
    outside = torch.from_numpy(buckets < 0).cuda()[:, None]
    for bad in (math.nan, math.inf):
        dirty = grad.masked_fill(outside, bad)
        assert torch.equal(bias.backward(dirty, 0, dtype=torch.float32), want)
        got = bias.add_to(dirty, 0, out=torch.empty_like(dirty))
        masked = outside.expand_as(got).clone()
        masked[:, 0] |= torch.from_numpy(buckets == 3).cuda()
        assert bool((got[masked] == -math.inf).all()) and bool(got[~masked].isfinite().all())
    grad[1, 1, 5, 2] = math.nan                      # distance -3, bucket 3 of head 1 alone
    got = bias.backward(grad, 0, dtype=torch.float32)
    assert bool(got[3, 1].isnan()) and int(got.isnan().sum()) == 1


def test_rows_without_any_bucket():
    """A sequence whose first key lies behind all of its queries: everything masked."""
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("causal")
    bias = tt.PositionBias(_normal(1, (n, 2), "float32"), of.cuda(), fill=-math.inf)
    offset = torch.tensor([0, 1000], device="cuda")
    got = bias.forward(30, 30, offset)
    assert bool((got[1] == -math.inf).all()) and bool(got[0].diagonal(0, 1, 2).isfinite().all())
    grad = _normal(2, (2, 2, 30, 30), "float32")
    assert torch.equal(bias.backward(grad, offset), bias.backward(grad[:1], 0))


def test_nothing():
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    bias = tt.PositionBias(_normal(1, (n, 2), "float32"), of.cuda())
    for size in ((0, 2, 3, 4), (1, 2, 0, 4), (1, 2, 3, 0)):
        grad = torch.empty(size, device="cuda")
        assert bias.forward(size[2], size[3], out=grad) is grad
        room = torch.full((n, 2), 3.0, device="cuda")
        assert bool((bias.backward(grad, 0, out=room, add=True) == 3.0).all())
        assert bool((bias.backward(grad, 0, out=room) == 0.0).all())


def test_offsets_beyond_32_bits():
    """4.4e9 scores in bf16: the last sequence's bias and gradient."""
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    bias = tt.PositionBias(_normal(1, (n, 2), "bfloat16"), of.cuda())
    batch, queries, keys = 130, 4100, 4100
    out = bias.forward(queries, keys, 0, out=torch.empty((batch, 2, queries, keys), dtype=torch.bfloat16, device="cuda"))
    one = bias.forward(queries, keys, 0)
    assert torch.equal(out[-1:], one) and torch.equal(out[:1], one)
    out.zero_()
    out[-1:] = _normal(2, (1, 2, queries, keys), "bfloat16")
    want = bias.backward(out[-1:], 0, dtype=torch.float32)
    got = bias.backward(out, 0, dtype=torch.float32)
    # the same values, and zeros, through other parts: 16.8e6 values for a head, of magnitude 0.8, and less than 10^4 additions each
    limit = 2 * 0.9 * queries * keys * 2.0 ** -24 * 1e4
    assert (got - want).abs().max() <= limit
    offsets = torch.zeros(batch, dtype=torch.int64, device="cuda")
    assert (bias.backward(out, offsets, dtype=torch.float32) - want).abs().max() <= limit
    out[-1:] = torch.randint(-2, 3, (1, 2, queries, keys), generator=torch.Generator().manual_seed(3)).bfloat16()
    want = bias.backward(out[-1:], 0, dtype=torch.float32)
    assert torch.equal(bias.backward(out, 0, dtype=torch.float32), want)      # sums of whole numbers, below 2^24 for a part
    assert torch.equal(bias.backward(out, offsets, dtype=torch.float32), want)


def test_graph_and_streams():
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    for size, ragged in (((2, 3, 200, 300), True), ((4, 2, 64, 700), False)):
        batch, heads, queries, keys = size
        table = _normal(1, (n, heads), "bfloat16")
        bias, eager = (tt.PositionBias(table, of.cuda()) for _ in range(2))
        scores, offset = _normal(2, size, "bfloat16"), torch.zeros(batch, dtype=torch.int64, device="cuda") if ragged else -100

        def step(b):
            return [b.forward(queries, keys, offset), b.add_to(scores, offset, out=torch.empty_like(scores)),
                    b.backward(scores, offset)]

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step(bias)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step(bias)
        bias.backward(_normal(1, (1, heads, 900, 900), "float32"))      # a larger workspace does not move the graph's
        for k in range(4):
            scores.copy_(_normal(3 + k, size, "bfloat16"))
            if ragged:
                offset.copy_(torch.tensor([-k, 40 * k - 60]))
            table.mul_(1.25)
            graph.replay()
            want = step(eager)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_weight_is_taken_as_it_is_at_a_call():
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    bias = tt.PositionBias(_normal(1, (n, 2), "float32"), of.cuda())
    bias.weight = _normal(2, (n, 5), "bfloat16")
    assert torch.equal(bias.forward(3, 200), tt.PositionBias(bias.weight, of.cuda()).forward(3, 200))


def test_refusals():
    import torch
    import paper_2206_10581_amd as tt
    of, n = _map("both")
    table = _normal(1, (n, 2), "float32")
    for bad in (of, of.cuda().long(), of.cuda()[1:], of.cuda()[None], of.cuda().repeat(3)[::3], of.cuda()[:0]):
        with pytest.raises(ValueError):
            tt.PositionBias(table, bad)
    with pytest.raises(ValueError):
        tt.PositionBias(table.cpu(), of)
    with pytest.raises(ValueError):
        tt.PositionBias(table, of.cuda(), fill=math.nan)
    bias, scores = tt.PositionBias(table, of.cuda()), _normal(2, (3, 2, 8, 16), "float32")
    offset = torch.zeros(3, dtype=torch.int64, device="cuda")
    bad = [lambda: bias.backward(scores[0]), lambda: bias.backward(scores.cpu()), lambda: bias.backward(scores[:, :1]),
           lambda: bias.backward(scores.transpose(2, 3)), lambda: bias.backward(scores, offset[:2]),
           lambda: bias.backward(scores, offset.int()), lambda: bias.backward(scores, offset.cpu()),
           lambda: bias.backward(scores, add=True), lambda: bias.backward(scores, out=table[:5]),
           lambda: bias.backward(scores.double()), lambda: bias.add_to(scores, out=scores[:, :, :4]),
           lambda: bias.add_to(scores[:1].expand(3, 2, 8, 16)), lambda: bias.add_to(scores, out=scores[:1].expand(3, 2, 8, 16)),
           lambda: bias.forward(8, 16, out=scores[:, :, :, :15]), lambda: bias.forward(8, 16, offset, out=scores[:2]),
           lambda: bias.forward(8, 16, out=scores, dtype=torch.bfloat16), lambda: bias.backward(scores, out=table, dtype=torch.half)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
