"""The gradient of a plain table by sorted ids, batches of more than 1024 positions: sums of several positions in every
type and piece, runs against the borders of tiles, sums added to what is there, strided tables, special values,
streams and graphs.

Tolerances.  u(type): half a unit of the last place of 1.  A tile has 8 or 16 sorted positions and adds up at most 32 (its
own and, where its last run ends there, the next tile's).  The parts of a longer run are added by two groups of
lanes or more, one after the other within a group: of at most 64 parts 32 each, of more ones m / 8 parts over 32
groups or more; then at most 6 additions join the lanes and 15 the wavefronts.  So a path through the additions of m
positions has at most min(m - 1, 32 + 33 + 6 + 15 + m / 256) of them, each with relative error 2^-24.  Then come the scale (or its
fused product and sum with what is there), 2^-24, and the rounding to the table's type, u."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}  # smallest steps of the types
TYPES = ["float32", "bfloat16", "float16"]


def _matrix(seed, rows, cols, kind, gap=0, lead=0):
    """Normal values, the flat buffer that they lie in, and which of its values are others'."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(lead + rows * (cols + gap) + 8, generator=g, device="cuda").to(getattr(torch, kind))
    m = flat[lead:lead + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    return m, flat


def _ids(seed, rows, B, hot=0.4, none=0.1):
    """One id in `hot` of the places, Zipf's law in most others, places without an id."""
    import torch
    rng = np.random.default_rng(seed)
    ids = np.minimum(np.exp(rng.random(B) * np.log(rows + 1)).astype(np.int64) - 1, rows - 1)
    ids = ids * 7 % rows if rows % 7 else ids
    ids[rng.random(B) < hot] = rows // 2
    empty = rng.random(B) < none
    ids[empty] = rng.choice([-1, rows, np.iinfo(np.int64).max, np.iinfo(np.int64).min], empty.sum())
    return torch.from_numpy(ids).cuda()


def _sums(ids, grad, rows, padding=-1):
    """Per id: the sum of its rows, of their magnitudes, and how many there are, in 64 bits."""
    import torch
    keep = torch.nonzero((ids >= 0) & (ids < rows) & (ids != padding))[:, 0]
    at, g = ids[keep], grad[keep].double()
    if len(ids) > 1_000_000:       # on the host: additions into one row wait for each other on the GPU
        columns = [[np.bincount(at.cpu(), weights=c, minlength=rows) for c in m.t().cpu().numpy()] for m in (g, g.abs())]
        total, size = (torch.from_numpy(np.stack(c, 1)).cuda() for c in columns)
        return total, size, torch.bincount(at, minlength=rows).double()[:, None]
    total = torch.zeros(rows, grad.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, g)
    size = torch.zeros_like(total).index_add_(0, at, g.abs())
    return total, size, torch.bincount(at, minlength=rows).double()[:, None]


def _check(got, total, size, count, scale, kind, base=None):
    import torch
    ref = scale * total + (0.0 if base is None else base)
    adds = torch.minimum((count - 1).clamp(min=0), 86 + count / 256)
    error = abs(scale) * size * adds * 2.0 ** -24 * 1.001 + 2.0 ** -24 * ref.abs()
    limit = error * (1 + U[kind]) + U[kind] * ref.abs() + TINY[kind]
    over = (got.double() - ref).abs() - limit
    assert got.isfinite().all() and over.max().item() <= 0, over.max().item()


def _both(rows, dim, B, kind, out_kind, gap=0, lead=0, scale=-0.75, seed=0, hot=0.4):
    """Written over what was there, and added to it; the values between the rows stay."""
    import torch
    import paper_2206_10581_amd as tt
    ids = _ids(seed + B, rows, B, hot)
    grad, _ = _matrix(seed + 1, B, dim, kind, gap, lead)
    total, size, count = _sums(ids, grad, rows)
    out, flat = _matrix(seed + 2, rows, dim, out_kind, gap, lead)
    kept = flat.clone()
    emb = tt.DenseEmbedding(out, B, scale=scale)
    base = out.double()
    emb.backward(ids, grad, out=out, add=True)
    _check(out, total, size, count, scale, out_kind, base)
    assert torch.equal(out.double()[count[:, 0] == 0], base[count[:, 0] == 0])
    out.fill_(float("nan"))
    emb.backward(ids, grad, out=out)
    _check(out, total, size, count, scale, out_kind)
    again = emb.backward(ids, grad, out=torch.empty_strided(out.shape, (dim, 1), dtype=out.dtype, device="cuda"))
    assert torch.equal(again, out)      # a fixed order
    out.copy_(kept[lead:lead + rows * (dim + gap)].view(rows, dim + gap)[:, :dim])
    assert torch.equal(flat, kept)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out_kind", TYPES)
@pytest.mark.parametrize("dim", [1, 8, 24, 63, 64, 65, 128, 129, 200, 257, 1001])
@pytest.mark.parametrize("B,gap,lead", [(1025, 0, 0), (5003, 3, 1), (13_001, 8, 0)])
def test_types_and_widths(kind, out_kind, dim, B, gap, lead):
    """Pieces of 1, 2, 4 and 8 values, rows that end inside one, runs of up to some 5000 positions, both kinds of sort."""
    _both(1009, dim, B, kind, out_kind, gap, lead)


@pytest.mark.parametrize("kind,out_kind", [("bfloat16", "float32"), ("float32", "bfloat16"), ("float16", "float16")])
@pytest.mark.parametrize("B,rows,dim", [
    (8192, 3001, 2048),                      # two micro-batches' shape; tiles of 8
    (8200, 1201, 4096),                      # tiles of 16 in 16-bit types by the number of pieces
    (32_768, 5003, 24), (32_769, 5003, 8), (32_769, 5003, 24), (40_001, 5003, 63),    # groups of lanes from 32,769 on
    (65_535, 5003, 65), (65_536, 5003, 65), (70_001, 5003, 130), (66_000, 907, 500),  # tiles of 16 by the number of ids
    (2_200_003, 50_021, 4),                  # more tiles than the blocks of a launch look at once
])
def test_sizes(kind, out_kind, B, rows, dim):
    _both(rows, dim, B, kind, out_kind, seed=3)


@pytest.mark.parametrize("B", [1500, 12_289, 16_385, 33_000])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,dim,gap,lead", [(1, 40, 8, 1), (2, 3, 1, 0), (70_001, 3, 5, 1), (70_001, 8, 1, 0), (30_011, 70, 2, 3)])
def test_strided_tables(B, kind, rows, dim, gap, lead):
    """Cleared row by row, in one launch or in shares of several; rows of fewer bytes than a piece among them."""
    _both(rows, dim, B, "bfloat16", kind, gap, lead, seed=5)


# Lengths of runs at the borders of tiles of 8 and 16, of two and three of them, and of 64 parts
LENGTHS = [1, 2, 7, 8, 9, 15, 16, 17, 18, 23, 24, 25, 31, 32, 33, 34, 47, 48, 49, 63, 64, 65, 127, 128, 129, 496, 503, 504, 505, 511, 512,
           513, 519, 520, 521, 1007, 1008, 1009, 1016, 1023, 1024, 1025, 1040, 1041, 2500, 9000]


@pytest.mark.parametrize("dim,kind,out_kind", [(65, "bfloat16", "float32"), (300, "float16", "float32"), (12, "float32", "float32"),
                                               (140, "float32", "bfloat16")])
@pytest.mark.parametrize("most", [3000, 50_000, 120_000])
@pytest.mark.parametrize("add", [False, True])
def test_runs_at_the_borders_of_tiles(dim, kind, out_kind, most, add):
    """Whole numbers whose sums are exact in any order: every position is counted once."""
    import torch
    import paper_2206_10581_amd as tt
    rng = np.random.default_rng(most + dim)
    lengths = []
    while sum(lengths) < 1025 or (sum(lengths) < most and len(lengths) < 4000):
        lengths.append(int(rng.choice(LENGTHS[:30] if most < 10_000 else LENGTHS)))
    first = int(rng.integers(0, 16))       # a short run in front moves all borders
    ids = rng.permutation(np.repeat(np.arange(len(lengths) + 1), [first, *lengths]))
    B, rows = len(ids), len(lengths) + 3
    ids = torch.from_numpy(ids).cuda()
    grad = torch.from_numpy(rng.integers(-4, 5, (B, dim)).astype(np.float32)).cuda().to(getattr(torch, kind))
    out = torch.from_numpy(rng.integers(-4, 5, (rows, dim)).astype(np.float32)).cuda().to(getattr(torch, out_kind))
    want = torch.zeros(rows, dim, dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double())
    if add:
        want += out.double()
    assert want.abs().max() < 2 ** 24
    got = tt.DenseEmbedding(out, B).backward(ids, grad, out=out, add=add)
    assert torch.equal(got, want.float().to(out.dtype))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("B,rows,dim", [(2000, 300, 40), (5003, 300, 300), (20_000, 3000, 130), (40_000, 3000, 20)])
@pytest.mark.parametrize("add", [False, True])
def test_special_values_stay_in_their_rows(kind, B, rows, dim, add):
    """Infinities and NaN reach the sums of their own ids alone, and none comes from positions without an id or with
    the padding's, though all of these lie in the same tiles."""
    import torch
    import paper_2206_10581_amd as tt
    ids = torch.randint(5, rows, (B,), generator=torch.Generator().manual_seed(B)).cuda()
    grad, _ = _matrix(4, B, dim, kind)
    ids[7::50], ids[9::50], ids[11::50], ids[13::50] = 0, 2, -1, 4
    grad[7::50], grad[9::50], grad[11::50], grad[13::50] = float("inf"), float("nan"), float("nan"), -float("inf")
    table = torch.ones((rows, dim), dtype=getattr(torch, kind), device="cuda")
    got = tt.DenseEmbedding(table, B, padding_id=4).backward(ids, grad, out=table, add=add)
    assert (got[0] == float("inf")).all() and got[2].isnan().all()
    assert (got[4] == (1.0 if add else 0.0)).all()
    keep = [k for k in range(rows) if k not in (0, 2)]
    assert got[keep].isfinite().all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("B,rows,dim", [(1500, 200, 136), (9000, 2003, 72), (20_001, 50_021, 40)])
def test_padding_and_update(kind, B, rows, dim):
    """The rows of the batch's ids, stepped in place; the padding's row and all others keep their bits."""
    import torch
    import paper_2206_10581_amd as tt
    ids = _ids(1, rows, B)
    weight, _ = _matrix(2, rows, dim, kind, 4, 2)
    grad, _ = _matrix(3, B, dim, kind)
    pad = rows // 2          # the id that most positions have
    emb = tt.DenseEmbedding(weight, B, scale=2.0, padding_id=pad)
    got = emb.backward(ids, grad, dtype=torch.float32)
    total, size, count = _sums(ids, grad, rows, pad)
    _check(got, total, size, count, 2.0, "float32")
    before = weight.clone()
    emb.backward_update(ids, grad, 0.125)
    _check(weight, total, size, count, -0.25, kind, before.double())
    still = count[:, 0] == 0
    assert still[pad] and torch.equal(weight[still], before[still]) and not torch.equal(weight, before)


@pytest.mark.parametrize("B,rows,dim", [(3000, 3000, 72), (20_000, 40_009, 24), (70_000, 4001, 65)])
def test_streams_and_graph(B, rows, dim):
    import torch
    import paper_2206_10581_amd as tt
    weight, _ = _matrix(1, rows, dim, "bfloat16")
    grad, _ = _matrix(2, B, dim, "bfloat16")
    grad = grad.contiguous()
    ids = _ids(3, rows, B)
    emb = tt.DenseEmbedding(weight, B, scale=2.0)
    sums = emb.backward(ids, grad).clone()
    into = torch.empty_like(sums)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        emb.backward(ids, grad, out=into)
    side.synchronize()
    assert torch.equal(into, sums)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emb.backward(ids, grad, out=into)
        emb.backward(ids, grad, out=into, add=True)
    for seed in (5, 6, 7):
        ids.copy_(_ids(seed, rows, B))
        grad.copy_(_matrix(seed, B, dim, "bfloat16")[0])
        into.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        sums = emb.backward(ids, grad)
        assert torch.equal(into, emb.backward(ids, grad, out=sums, add=True))


def test_a_table_without_rows():
    """Every id is outside it."""
    import torch
    import paper_2206_10581_amd as tt
    for B in (0, 5, 2000):
        emb = tt.DenseEmbedding(torch.empty(0, 24, device="cuda"), 2000)
        ids = torch.arange(B, device="cuda") - 2
        grad = torch.ones(B, 24, device="cuda")
        out = torch.full((B, 24), float("nan"), device="cuda")
        assert not emb.forward(ids, out=out).any() and emb.backward(ids, grad).shape == (0, 24)
        emb.backward_update(ids, grad, 1.0)
