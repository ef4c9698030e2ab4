"""The norm of many tensors and clipping, against numpy in 64 bits.

Tolerances.  Squares and sums are in fp64, so the norm's error is its rounding to fp32, 2^-24, and n * 2^-52 for a sum
of n squares.  A clipped value is a product that is rounded to fp32 and to its type, 2^-24 + u(type); the tests allow
a second rounding in fp32, that of the factor."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}
SIZES = {
    "one": [1],
    "few": [5, 0, 2048, 2049, 7, 100_003],
    "empty": [0, 0],
    "many": [(37 * k) % 3001 for k in range(300)],     # several launches' lists, some of them empty
    "border": [9] * 96 + [0] * 96 + [2047] * 96,
    "long": [3_000_001, 1, 5_000_000],
}


def _tensors(sizes, kinds, seed, scale=1.0):
    """Tensors one behind the other in a buffer per type, so that most start at odd places."""
    import torch
    g = torch.Generator().manual_seed(seed)
    kind = [kinds[k % len(kinds)] for k in range(len(sizes))]
    flat = {k: (torch.randn(1 + sum(n for n, t in zip(sizes, kind) if t == k), generator=g) * scale)
            .to(getattr(torch, k)).cuda() for k in kinds}
    at, found = dict.fromkeys(kinds, 1), []
    for n, k in zip(sizes, kind):
        found.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    return found


def _norm(tensors, scale=1.0):
    total = sum(float((t.double().cpu().numpy() ** 2).sum()) for t in tensors)
    return abs(scale) * np.sqrt(total), sum(t.numel() for t in tensors)


def _near(got, ref, n):
    assert abs(got.item() - ref) <= ref * (2.0 ** -24 + n * 2.0 ** -52) + 2.0 ** -150, (got.item(), ref)


KINDS = [["float32"], ["bfloat16"], ["float16"], ["float32", "bfloat16", "float16"]]


@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES.keys())
@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
def test_norm(sizes, kinds):
    import paper_2206_10581_amd as tt
    tensors = _tensors(sizes, kinds, 1)
    clip = tt.GradientClip(tensors)
    for scale in (1.0, -0.25):
        _near(clip.norm(scale=scale), *_norm(tensors, scale))
    assert clip.norm().item() == clip.norm().item()


@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES.keys())
@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
@pytest.mark.parametrize("out", ["place", "float32", "bfloat16", "float16"])
@pytest.mark.parametrize("limit,scale", [(0.5, 1.0), (0.5, 0.125), (2.0, 1.0), (2.0, -0.5), (0.0, 1.0)])
def test_clip(sizes, kinds, out, limit, scale):
    """limit: the largest norm, in norms."""
    import torch
    import paper_2206_10581_amd as tt
    tensors = _tensors(sizes, kinds, 2)
    before = [t.clone() for t in tensors]
    norm, n = _norm(before, scale)
    outs = None if out == "place" else [torch.full_like(t, float("nan"), dtype=getattr(torch, out)) for t in tensors]
    max_norm = float(np.float32(limit * norm))
    got = tt.GradientClip(tensors, out=outs).clip(max_norm, scale=scale, eps=1e-6)
    _near(got, norm, n)
    factor = scale * min(1.0, max_norm / (norm + float(np.float32(1e-6))))
    for was, now, kept in zip(before, tensors if outs is None else outs, tensors):
        ref = was.double().cpu().numpy() * factor
        kind = str(now.dtype).split(".")[1]
        err = np.abs(now.double().cpu().numpy() - ref)
        assert (err <= np.abs(ref) * (2 * 2.0 ** -24 + U[kind] + n * 2.0 ** -52) + TINY[kind]).all()
        if outs is not None or factor == 1.0:
            assert torch.equal(kept, was)


@pytest.mark.parametrize("size", [1e30, 1e-30, 1e-42])
def test_squares_beyond_fp32(size):
    import paper_2206_10581_amd as tt
    tensors = _tensors([1000, 3, 20_000], ["float32"], 3, size)
    clip = tt.GradientClip(tensors)
    norm, n = _norm(tensors)
    _near(clip.norm(), norm, n)
    clip.clip(norm / 4, eps=0.0)
    after, _ = _norm(tensors)
    assert abs(after - norm / 4) <= norm / 4 * 1e-6 + 2.0 ** -149 * np.sqrt(n)


def test_a_norm_beyond_fp32_still_clips():
    import torch
    import paper_2206_10581_amd as tt
    x = torch.full((4096,), 3e38, device="cuda")
    assert tt.GradientClip([x]).clip(1.0).item() == float("inf")
    assert torch.allclose(x, torch.full_like(x, 1 / 64), rtol=1e-6, atol=0)


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_values_that_are_not_finite_are_not_hidden(kind, bad):
    import torch
    import paper_2206_10581_amd as tt
    tensors = _tensors([50, 4000], [kind], 4)
    tensors[1][3999] = bad
    norm = tt.GradientClip(tensors).clip(1.0)
    if np.isnan(bad):
        assert norm.isnan() and all(t.isnan().all() for t in tensors)
    else:
        assert norm.item() == float("inf")
        assert not tensors[0].any() and not tensors[1][:3999].any() and tensors[1][3999].isnan()
    same = _tensors([50, 4000], [kind], 4)
    same[1][3999] = bad
    assert torch.equal(tt.GradientClip(same).norm().isnan(), norm.isnan())


def test_orders_of_dimensions():
    import torch
    import paper_2206_10581_amd as tt
    a = torch.randn(6, 50, 7, device="cuda")
    tensors = [a.permute(2, 0, 1), a[:0], torch.tensor(2.0, device="cuda"), torch.randn(1, 9, 1, device="cuda").expand(1, 9, 1)]
    _near(tt.GradientClip(tensors).norm(), *_norm(tensors))
    outs = [torch.empty_like(t) for t in tensors]
    want = [t.clone() for t in tensors]
    tt.GradientClip(tensors, out=outs).clip(1e9)
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_tensors_beyond_32_bits():
    import torch
    import paper_2206_10581_amd as tt
    n = (1 << 31) + 12_345
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    clip = tt.GradientClip([x[:5], x])
    _near(clip.norm(), np.sqrt(n + 5.0), n)
    tt.GradientClip([x]).clip(float(np.sqrt(n) / 2), eps=0.0)
    assert all((part == 0.5).all() for part in x.split(1 << 28))


def test_streams_and_graph():
    import torch
    import paper_2206_10581_amd as tt
    tensors = _tensors(SIZES["many"], ["float32", "bfloat16"], 6)
    outs = [torch.empty_like(t, dtype=torch.float32) for t in tensors]
    clip = tt.GradientClip(tensors, out=outs)
    want = clip.clip(3.0).item()
    first = [t.clone() for t in outs]
    norm = torch.empty((), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        [t.fill_(float("nan")) for t in outs]
        clip.clip(3.0, out=norm)
    side.synchronize()
    assert norm.item() == want and all(torch.equal(x, y) for x, y in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip.clip(3.0, out=norm)
    for factor in (2.0, 0.001, 30.0):
        [t.mul_(factor) for t in tensors]
        graph.replay()
        torch.cuda.synchronize()
        got, kept = norm.item(), [t.clone() for t in outs]
        assert got == clip.clip(3.0).item() and all(torch.equal(x, y) for x, y in zip(kept, outs))


def test_refusals():
    import torch
    import paper_2206_10581_amd as tt
    x = torch.zeros(8, 8, device="cuda")
    for bad in (lambda: tt.GradientClip([]), lambda: tt.GradientClip([x.cpu()]), lambda: tt.GradientClip([x, x.cpu()]),
                lambda: tt.GradientClip([x.double()]), lambda: tt.GradientClip([x[:, :4]]),
                lambda: tt.GradientClip([x[:1].expand(8, 8)]), lambda: tt.GradientClip([x], out=[x[:4]]),
                lambda: tt.GradientClip([x], out=[x.t()]), lambda: tt.GradientClip([x], out=[x, x]),
                lambda: tt.GradientClip([x]).norm(out=x), lambda: tt.GradientClip([x]).norm(out=torch.zeros(()))):
        with pytest.raises(ValueError):
            bad()
    clip = tt.GradientClip([x])
    for bad in (lambda: clip.clip(-1.0), lambda: clip.clip(float("nan")), lambda: clip.clip(1.0, eps=-1.0),
                lambda: clip.norm(scale=float("inf")), lambda: clip.clip(1.0, scale=float("nan"))):
        with pytest.raises(tt.TTEmbError):
            bad()


def test_the_memory_of_replaced_tensors_is_held():
    """The object works on the memory that the tensors had when it was made, which is not given to others."""
    import torch
    import paper_2206_10581_amd as tt
    x, y = torch.full((100_000,), 3.0, device="cuda"), torch.zeros(100_000, device="cuda")
    clip = tt.GradientClip([x], out=[y])
    x.data, y.data = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    others = [torch.full((100_000,), 7.0, device="cuda") for _ in range(4)]
    want = 3.0 * 100_000 ** 0.5
    assert abs(clip.clip(1.0).item() - want) <= want * 2.0 ** -23
    assert all(bool((t == 7.0).all()) for t in others)
