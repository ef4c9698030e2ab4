"""Plain tables: lookup with a scale and gradient by sorted ids, against plain sums in 64 bits.

Tolerances.  u(type) is half a unit of the last place of 1: 2^-24 for fp32, 2^-8 for bf16, 2^-11 for fp16.  A lookup is
one product in fp32 and one rounding to the output's type: relative error 2^-24 + u.  A sum of m values: up to 1024
positions are added by eights, at most 8 + 32 + 4 additions in fp32 touching a value.  More are cut into tiles of 8 or 16
sorted positions, of which a tile adds up at most 32; the parts of a longer run, m/8 and two more, are added one after
the other by two groups of lanes (of more than 64 parts by 32 groups) and joined in 6 + 15 more.  The tests allow
64 + m/32 additions, which is no fewer: 32 + (m/16 + 1) + 6 to 496 positions, 32 + 32 + 6 to where 64 parts end, and
32 + (m/256 + 1) + 21 beyond.  Each has relative error 2^-24; then come the scale (2^-24) and the output's rounding."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}  # smallest steps of the types
TYPES = ["float32", "bfloat16", "float16"]


def _torch(kind):
    import torch
    return getattr(torch, kind)


def _normal(seed, shape, kind, gap=0, lead=0):
    """Normal values on the GPU; gap: unused columns behind every row, lead: unused values in front of the first."""
    import torch
    g = torch.Generator().manual_seed(seed)
    flat = torch.randn(lead + shape[0] * (shape[1] + gap), generator=g).to(_torch(kind)).cuda()
    return flat[lead:].view(shape[0], shape[1] + gap)[:, :shape[1]]


def _ids(seed, rows, B, how):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, rows, B)
    if how == "one":
        ids[:] = rows - 1
    elif how == "none":
        ids[:] = np.where(rng.random(B) < 0.5, -1, rows)
    elif how == "hot":        # a run over many tiles, some empty places of every kind
        ids[rng.random(B) < 0.6] = rows // 2
        ids[rng.random(B) < 0.1] = -1
        ids[rng.random(B) < 0.05] = np.iinfo(np.int64).max
        ids[rng.random(B) < 0.05] = np.iinfo(np.int64).min
    elif how == "runs":       # runs of lengths that start and end all over the tiles
        ids = np.repeat(np.arange(B) % rows, rng.integers(1, 130, B))[:B]
        ids = rng.permutation(ids)
    return ids


def _sums(ids, grad, rows, padding=-1):
    """Per id: the sum of its rows, of their magnitudes, and how many there are, in 64 bits."""
    g = grad.double().cpu().numpy()
    keep = (ids >= 0) & (ids < rows) & (ids != padding)
    total, size, count = (np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1])), np.zeros(rows))
    np.add.at(total, ids[keep], g[keep])
    np.add.at(size, ids[keep], np.abs(g[keep]))
    np.add.at(count, ids[keep], 1)
    return total, size, count


def _check(got, ref, bound, kind):
    got = got.double().cpu().numpy()
    limit = bound + U[kind] * np.abs(ref) + TINY[kind]
    worst = np.max(np.abs(got - ref) - limit, initial=-1.0)
    assert np.isfinite(got).all() and worst <= 0, worst


def _bound(size, count, scale):
    return abs(scale) * size * (64 + count[:, None] / 32 + 2) * 2.0 ** -24


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out_kind", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 7, 8, 9, 64, 100, 513, 2056])
def test_lookup(kind, out_kind, dim):
    import torch
    import paper_2206_10581_amd as tt
    for B, gap, lead in ((1, 0, 0), (77, 3, 1), (1030, 0, 5)):
        table = _normal(B, (211, dim), kind, gap, lead)
        ids = _ids(B, 211, B, "hot")
        emb = tt.DenseEmbedding(table, B, scale=1.7)
        wide = torch.full((B, dim + 2), 7.0, dtype=_torch(out_kind), device="cuda")
        got = emb.forward(torch.from_numpy(ids).cuda(), out=wide[:, 1:1 + dim])
        inside = (ids >= 0) & (ids < 211)
        ref = table.double().cpu().numpy()[np.where(inside, ids, 0)] * float(np.float32(1.7)) * inside[:, None]
        _check(got, ref, 2.0 ** -24 * np.abs(ref), out_kind)
        assert not got[torch.from_numpy(~inside).cuda()].any()
        assert (wide[:, 0] == 7.0).all() and (wide[:, -1] == 7.0).all()   # its columns only


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out_kind", TYPES)
@pytest.mark.parametrize("dim", [1, 5, 8, 63, 129, 1000])
@pytest.mark.parametrize("add", [False, True])
def test_gradient_types_and_widths(kind, out_kind, dim, add):
    import torch
    import paper_2206_10581_amd as tt
    rows, scale = 97, -0.75
    for B, how, gap, lead in ((1, "uniform", 0, 0), (64, "hot", 1, 3), (700, "hot", 8, 0)):
        ids = _ids(B + dim, rows, B, how)
        grad = _normal(dim, (B, dim), kind, gap, lead)
        emb = tt.DenseEmbedding(torch.zeros((rows, dim), dtype=_torch(out_kind), device="cuda"), B, scale=scale)
        out = _normal(dim + 1, (rows, dim), out_kind, gap, lead)
        base = out.double().cpu().numpy() if add else 0.0
        got = emb.backward(torch.from_numpy(ids).cuda(), grad, out=out, add=add)
        total, size, count = _sums(ids, grad, rows)
        ref = base + scale * total
        _check(got, ref, _bound(size, count, scale) + 2.0 ** -24 * np.abs(ref), out_kind)
        if add:
            untouched = count == 0
            assert (got.double().cpu().numpy()[untouched] == base[untouched]).all()


@pytest.mark.parametrize("rows", [1, 2, 40, 2048, 30_011, 3_000_017])
@pytest.mark.parametrize("B,how", [(0, "uniform"), (1, "one"), (31, "one"), (32, "one"), (33, "one"), (65, "one"),
                                   (96, "one"), (97, "one"), (1000, "none"), (1001, "hot"), (5000, "runs"),
                                   (20_000, "one"), (20_003, "runs"), (20_003, "uniform")])
def test_gradient_runs(rows, B, how):
    """Runs of every length against the borders of tiles; row counts with one, two and three digits of a sort."""
    import torch
    import paper_2206_10581_amd as tt
    dim = 12
    ids = _ids(B + rows, rows, B, how)
    grad = _normal(B, (B, dim), "float32")
    emb = tt.DenseEmbedding(torch.zeros((rows, dim), device="cuda"), max(B, 1), scale=2.0)
    got = emb.backward(torch.from_numpy(ids).cuda(), grad, out=torch.full((rows, dim), float("nan"), device="cuda"))
    total, size, count = _sums(ids, grad, rows)
    _check(got, 2.0 * total, _bound(size, count, 2.0), "float32")
    assert torch.equal(got, emb.backward(torch.from_numpy(ids).cuda(), grad))     # a fixed order


@pytest.mark.parametrize("B,dim,kind", [(32_768, 3, "float16"), (32_768, 24, "bfloat16"), (32_769, 3, "float16"),
                                        (32_769, 24, "bfloat16"), (32_769, 63, "float32"), (65_535, 72, "bfloat16"), (65_536, 65, "float32"), (70_000, 480, "bfloat16"),
                                        (140_001, 8, "float32"), (530_003, 4, "bfloat16")])
def test_gradient_long_batches(B, dim, kind):
    import torch
    import paper_2206_10581_amd as tt
    rows = 70_001
    ids = _ids(5, rows, B, "hot")
    grad = _normal(5, (B, dim), kind)
    emb = tt.DenseEmbedding(torch.zeros((rows, dim), device="cuda"), B)
    got = emb.backward(torch.from_numpy(ids).cuda(), grad)
    total, size, count = _sums(ids, grad, rows)
    _check(got, total, _bound(size, count, 1.0), "float32")


@pytest.mark.parametrize("B", [1, 2, 8, 9, 33, 64, 65, 500, 512, 513, 1023, 1024, 1025])
@pytest.mark.parametrize("rows", [1, 7, 31, 32, 33, 1000, 262_144, 262_145])
@pytest.mark.parametrize("how", ["uniform", "hot", "one", "none"])
def test_gradient_of_few_positions(rows, B, how):
    """Rows of three fp16 values: the cleared words hold parts of up to four rows, some of them with positions."""
    import torch
    import paper_2206_10581_amd as tt
    ids = _ids(B + rows, rows, B, how)
    d_ids = torch.from_numpy(ids).cuda()
    for dim, kind, lead, gap in ((3, "float16", 1, 0), (1, "bfloat16", 3, 0), (5, "float32", 1, 0), (9, "float16", 0, 4)):
        if rows > 1000 and gap == 0 and dim != 3:
            continue
        flat = torch.full((lead + rows * (dim + gap) + 9,), 7.0, dtype=_torch(kind), device="cuda")
        out = flat[lead:lead + rows * (dim + gap)].view(rows, dim + gap)[:, :dim]
        grad = _normal(dim, (B, dim), kind)
        emb = tt.DenseEmbedding(out, B, scale=0.5)
        got = emb.backward(d_ids, grad, out=out)
        total, size, count = _sums(ids, grad, rows)
        _check(got, 0.5 * total, _bound(size, count, 0.5), kind)
        base = got.double().cpu().numpy()
        _check(emb.backward(d_ids, grad, out=out, add=True), base + 0.5 * total,
               _bound(size, count, 0.5) + 2.0 ** -24 * np.abs(base + 0.5 * total), kind)
        out.fill_(7.0)
        assert (flat == 7.0).all()


@pytest.mark.parametrize("B", [1024, 1025, 2048, 2049, 4096, 4097, 6144, 6145, 8192, 8193, 10_240, 10_241, 12_288, 12_289,
                               16_384, 16_385])
@pytest.mark.parametrize("rows,dim", [(5003, 8), (2_900_001, 24)])
def test_gradient_sorts(rows, dim, B):
    """Batch sizes at which another sort takes over, beside tables that are cleared quickly and slowly."""
    import torch
    import paper_2206_10581_amd as tt
    ids = _ids(B, rows, B, "hot")
    grad = _normal(B, (B, dim), "float32")
    emb = tt.DenseEmbedding(torch.zeros((rows, dim), device="cuda"), B)
    got = emb.backward(torch.from_numpy(ids).cuda(), grad, out=torch.full((rows, dim), float("nan"), device="cuda"))
    total, size, count = _sums(ids, grad, rows)
    _check(got, total, _bound(size, count, 1.0), "float32")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,dim,gap,lead", [(1, 1, 0, 1), (1, 9, 4, 1), (3, 1, 0, 3), (301, 3, 0, 1), (301, 3, 2, 1),
                                               (77, 8, 1, 5), (77, 13, 0, 7), (40, 700, 3, 1), (5, 9001, 1, 3)])
@pytest.mark.parametrize("B", [0, 5])
def test_gradient_writes_every_row_and_nothing_else(rows, dim, gap, lead, kind, B):
    import torch
    import paper_2206_10581_amd as tt
    flat = torch.full((lead + rows * (dim + gap) + 11,), 7.0, dtype=_torch(kind), device="cuda")
    out = flat[lead:lead + rows * (dim + gap)].view(rows, dim + gap)[:, :dim]
    ids = _ids(B, rows, B, "uniform")
    grad = _normal(dim, (B, dim), "float32")
    got = tt.DenseEmbedding(out, max(B, 1)).backward(torch.from_numpy(ids).cuda(), grad, out=out)
    total, size, count = _sums(ids, grad, rows)
    _check(got, total, _bound(size, count, 1.0), kind)
    out.fill_(7.0)
    assert (flat == 7.0).all()


def test_gradient_of_padding_and_update():
    import torch
    import paper_2206_10581_amd as tt
    rows, dim, B = 50, 24, 300
    ids = _ids(1, rows, B, "hot")
    weight = _normal(2, (rows, dim), "float32")
    grad = _normal(3, (B, dim), "float32")
    emb = tt.DenseEmbedding(weight, B, scale=3.0, padding_id=rows // 2)
    d_ids = torch.from_numpy(ids).cuda()
    assert emb.forward(d_ids)[torch.from_numpy(ids == rows // 2).cuda()].any()    # padding has a row
    got = emb.backward(d_ids, grad)
    total, size, count = _sums(ids, grad, rows, rows // 2)
    _check(got, 3.0 * total, _bound(size, count, 3.0), "float32")
    assert not got[rows // 2].any()
    before = weight.double().cpu().numpy()
    emb.backward_update(d_ids, grad, 0.01)
    rate = float(np.float32(0.03))
    ref = before - rate * total
    _check(weight, ref, _bound(size, count, rate) + 2.0 ** -23 * (np.abs(ref) + rate * np.abs(total)), "float32")
    assert (weight.double().cpu().numpy()[count == 0] == before[count == 0]).all()


def test_gradient_is_that_of_the_lookup():
    """Differences of L = sum(upstream * forward(ids)) in every entry of the table; all numbers are whole, so they are exact."""
    import torch
    import paper_2206_10581_amd as tt
    rows, dim, B = 5, 3, 40
    rng = np.random.default_rng(0)
    weight = torch.from_numpy(rng.integers(-8, 9, (rows, dim)).astype(np.float32)).cuda()
    up = torch.from_numpy(rng.integers(-8, 9, (B, dim)).astype(np.float32)).cuda()
    ids = torch.from_numpy(rng.integers(-1, rows + 1, B)).cuda()
    emb = tt.DenseEmbedding(weight, B, scale=0.5)
    got = emb.backward(ids, up).clone()
    for v in range(rows):
        for j in range(dim):
            sides = []
            for step in (1.0, -1.0):
                weight[v, j] += step
                sides.append((up * emb.forward(ids)).double().sum().item())
                weight[v, j] -= step
            assert (sides[0] - sides[1]) / 2 == got[v, j].item()


@pytest.mark.parametrize("kind", TYPES)
def test_special_values_stay_in_their_rows(kind):
    """Infinities and NaN reach the sums of their own ids alone, and none comes from positions without an id."""
    import torch
    import paper_2206_10581_amd as tt
    rows, dim, B = 20, 40, 500
    ids = _ids(4, rows, B, "uniform")
    ids[7], ids[9], ids[11] = 3, 4, -1
    grad = _normal(4, (B, dim), kind)
    grad[7], grad[9], grad[11] = float("inf"), float("nan"), float("nan")
    emb = tt.DenseEmbedding(torch.zeros((rows, dim), dtype=_torch(kind), device="cuda"), B)
    got = emb.backward(torch.from_numpy(ids).cuda(), grad)
    assert got[4].isnan().all() and (got[3] == float("inf")).all()
    keep = torch.ones(rows, dtype=torch.bool)
    keep[3] = keep[4] = False
    assert got.cpu()[keep].isfinite().all()
    table = torch.ones((rows, dim), dtype=_torch(kind), device="cuda")
    table[0] = float("nan")
    out = tt.DenseEmbedding(table, 3).forward(torch.tensor([-1, 0, rows], device="cuda"))
    assert not out[0].any() and out[1].isnan().all() and not out[2].any()


def test_tables_beyond_32_bits():
    """Offsets beyond 2^32 bytes and 2^31 values in lookups and gradients."""
    import torch
    import paper_2206_10581_amd as tt
    rows, dim = 550_000, 4096
    table = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    last = rows - 1 - torch.arange(5, device="cuda")
    table[last] = _normal(1, (5, dim), "bfloat16")
    emb = tt.DenseEmbedding(table, 8)
    assert torch.equal(emb.forward(last), table[last])
    grad = _normal(2, (5, dim), "bfloat16")
    table.fill_(1.0)
    got = emb.backward(last, grad, out=table)
    assert torch.equal(got[last], grad)
    got[last] = 0
    assert all(not part.any() for part in got.split(50_000))


def test_streams_and_graph():
    import torch
    import paper_2206_10581_amd as tt
    rows, dim, B = 3000, 72, 900
    weight = _normal(1, (rows, dim), "bfloat16")
    grad = _normal(2, (B, dim), "bfloat16")
    ids = torch.from_numpy(_ids(3, rows, B, "hot")).cuda()
    emb = tt.DenseEmbedding(weight, B, scale=2.0)
    row, sums = emb.forward(ids).clone(), emb.backward(ids, grad).clone()
    out, into = torch.empty_like(row), torch.empty_like(sums)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        emb.forward(ids, out=out)
        emb.backward(ids, grad, out=into)
    side.synchronize()
    assert torch.equal(out, row) and torch.equal(into, sums)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emb.forward(ids, out=out)
        emb.backward(ids, grad, out=into)
        emb.backward(ids, grad, out=into, add=True)
    for seed in (5, 6, 7):
        ids.copy_(torch.from_numpy(_ids(seed, rows, B, "runs")).cuda())
        grad.copy_(_normal(seed, (B, dim), "bfloat16"))
        out.fill_(float("nan"))
        into.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        row, sums = emb.forward(ids), emb.backward(ids, grad)
        assert torch.equal(out, row) and torch.equal(into, emb.backward(ids, grad, out=sums, add=True))


def test_refusals():
    import torch
    import paper_2206_10581_amd as tt
    weight = torch.zeros((10, 16), device="cuda")
    emb = tt.DenseEmbedding(weight, 4)
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    grad = torch.zeros((4, 16), device="cuda")
    for bad in (lambda: emb.forward(ids.int()), lambda: emb.forward(ids.cpu()), lambda: emb.forward(ids[::2]),
                lambda: emb.forward(ids.view(2, 2)), lambda: emb.forward(ids, out=grad[:, :8]),
                lambda: emb.forward(ids, out=grad.t().contiguous().t()), lambda: emb.forward(ids, out=grad.double()),
                lambda: emb.forward(ids, out=grad, dtype=torch.float16), lambda: emb.backward(ids, grad[:3]),
                lambda: emb.backward(ids, grad.cpu()), lambda: emb.backward(ids, grad, out=weight[:9]),
                lambda: emb.backward(ids, grad, add=True), lambda: emb.backward(ids, grad[:1].expand(4, 16)),
                lambda: tt.DenseEmbedding(weight.cpu(), 4), lambda: tt.DenseEmbedding(weight.long(), 4),
                lambda: tt.DenseEmbedding(weight.t(), 4), lambda: tt.DenseEmbedding(weight[0], 4),
                lambda: tt.DenseEmbedding(weight[:, :0], 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: emb.forward(torch.zeros(5, dtype=torch.int64, device="cuda")),
                lambda: tt.DenseEmbedding(weight, 0), lambda: tt.DenseEmbedding(weight, 1 << 30)):
        with pytest.raises(tt.TTEmbError):
            bad()


def test_a_weight_whose_storage_is_replaced():
    """The table is looked for where it is at the time of a call."""
    import torch
    import paper_2206_10581_amd as tt
    weight = torch.nn.Parameter(_normal(1, (30, 8), "float32"), requires_grad=False)
    emb = tt.DenseEmbedding(weight, 4)
    ids = torch.tensor([3, 29, 0], device="cuda")
    assert torch.equal(emb.forward(ids), weight[ids])
    weight.data = _normal(2, (30, 8), "float32")
    assert torch.equal(emb.forward(ids), weight[ids])
    weight.data = _normal(3, (30, 8), "bfloat16")
    assert torch.equal(emb.forward(ids), weight[ids])
