"""Scores of logits, their gradient and the loss in one call, against plain forms in 64 bits.

Tolerances.  u = 2^-24.  The kernels hold y = (x - m) c, c = scale / log 2 and m the largest logit they have met: a difference, c's own
rounding and a product, 3 u |y|; 2^y by the hardware, 2 u (one unit of the last place).  A value then goes through the additions of a
thread's sum, those over 64 lanes and 16 wavefronts (6 + 4) and of 64 parts (6), and through a rescaling, three roundings and 2^y again,
whenever a larger logit turns up: ROUNDINGS counts, for V columns of at least 64 lanes with one or more, V / 64 additions, 16 for the joins
and 4 for each of up to 16 rescalings (a maximum of random logits rises about log V times; sorted ones are tested apart).
With Z = E|z| and ZZ = E z^2 over the row (z = log 2 y), log S is off by u (ROUNDINGS + 2 + 3 Z) and the logarithm's own
2 u |log S|; T / S likewise with |z| inside the mean; log p adds 3 u |z| and the rounding of the difference."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
# 2^y below 2^-126 is 0; its factors are a scale of up to 30 and |log p + entropy|, up to 126 log 2 + 11: together below 2^12
TINY = {"float32": 2.0 ** -114, "bfloat16": 2.0 ** -114, "float16": 2.0 ** -24}
TYPES = ["float32", "bfloat16", "float16"]
# narrow rows of every kind, both sides of each border, and wide ones with and without a rest
COLS = [1, 2, 3, 4, 7, 8, 10, 16, 17, 33, 47, 64, 65, 128, 129, 256, 257, 511, 513, 1024, 1025, 2048, 2049, 5000, 8192, 33_001]


def _logits(seed, shape, kind, gap=0, lead=0, spread=3.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    flat = (torch.randn(lead + shape[0] * (shape[1] + gap), generator=g) * spread).to(getattr(torch, kind)).cuda()
    return flat[lead:].view(shape[0], shape[1] + gap)[:, :shape[1]]


def _tokens(seed, rows, cols, pad=0.0):
    import torch
    rng = np.random.default_rng(seed)
    t = rng.integers(0, cols, rows)
    t[rng.random(rows) < pad / 2] = -100
    t[rng.random(rows) < pad / 2] = cols
    return torch.from_numpy(t).cuda()


class Reference:
    """The definitions in 64 bits, with what the tolerances need."""

    def __init__(self, logits, tokens, scale, roundings=None):
        import torch
        x, scale = logits.double(), float(np.float32(scale))
        rows, cols = x.shape
        self.x, self.scale, self.cols = x, scale, cols
        self.counts = torch.ones(rows, dtype=torch.bool, device="cuda") if tokens is None else (tokens >= 0) & (tokens < cols)
        self.at = torch.zeros(rows, dtype=torch.int64, device="cuda") if tokens is None else torch.where(self.counts, tokens, 0)
        most = x.amax(1, keepdim=True)
        self.empty = (most == -math.inf)[:, 0]
        z = (x - most.masked_fill(most == -math.inf, 0.0)) * scale
        e = z.exp()
        total = e.sum(1, keepdim=True)
        self.logs = total.log()
        self.logp = torch.where(self.empty[:, None], -math.inf, z - self.logs)
        self.p = torch.where(self.empty[:, None], 0.0, e / total)
        self.z = torch.where(e > 0, z, 0.0)
        self.h = torch.where(self.empty, 0.0, -(self.p * torch.where(self.p > 0, self.logp, 0.0)).sum(1))
        k = roundings if roundings is not None else cols / 64 + 16 + 4 * 16
        size, square = (self.p * self.z.abs()).sum(1), (self.p * self.z ** 2).sum(1)
        self.logs_tol = u * (k + 2 + 3 * size + 2 * self.logs[:, 0].abs().nan_to_num(0, 0, 0))
        self.h_tol = self.logs_tol * (1 + size) + u * ((k + 8) * size + 4 * square + 2 * self.h)
        self.logp_tol = self.logs_tol[:, None] + u * (3 * self.z.abs() + 2 * self.logp.abs().nan_to_num(0, 0, 0))

    def logprobs(self):
        import torch
        return (torch.where(self.counts, self.logp.gather(1, self.at[:, None])[:, 0], 0.0),
                self.logp_tol.gather(1, self.at[:, None])[:, 0])

    def entropy(self):
        import torch
        return torch.where(self.counts, self.h, 0.0), self.h_tol

    def top(self, k):
        import torch
        ids = self.x.sort(dim=1, descending=True, stable=True)[1][:, :k]
        values = self.logp.gather(1, ids)
        tol = self.logp_tol.gather(1, ids)
        if k > self.cols:
            more = k - self.cols
            ids = torch.nn.functional.pad(ids, (0, more), value=-1)
            values = torch.nn.functional.pad(values, (0, more), value=-math.inf)
            tol = torch.nn.functional.pad(tol, (0, more))
        out = ~self.counts[:, None]
        return ids.masked_fill(out, -1), values.masked_fill(out, -math.inf), tol

    def gradient(self, d, h):
        """The gradient, and the bound of its error before the last rounding.  p from the state: y takes 2 u |z| more for the
        state's logarithm and its conversion, and 2^y two units; then the factors, 6 u."""
        import torch
        hot = torch.zeros_like(self.x).scatter_(1, self.at[:, None], 1.0)
        d = torch.zeros_like(self.h) if d is None else d.double()
        h = torch.zeros_like(self.h) if h is None else h.double()
        keep = (self.counts & ~self.empty)[:, None]
        logp = torch.where(self.p > 0, self.logp, 0.0)
        g = self.scale * (d[:, None] * (hot - self.p) - h[:, None] * self.p * (logp + self.h[:, None]))
        size = self.scale * ((d[:, None] * hot).abs() + self.p * (d[:, None].abs() + h[:, None].abs() *
                                                                 (logp.abs() + self.h[:, None])))
        rel = self.logs_tol[:, None] + u * (12 + 5 * (self.z.abs() + self.logs.abs().nan_to_num(0, 0, 0)))
        tol = size * rel + self.scale * h[:, None].abs() * self.p * (self.h_tol + self.logs_tol)[:, None]
        return torch.where(keep, g, 0.0), tol


def _check(got, ref, tol, kind="float32"):
    import torch
    got = got.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    limit = tol + U[kind] * ref.abs() + TINY[kind]
    bad = ~(same | ((got - ref).abs() <= limit))
    if bool(bad.any()):
        at = tuple(bad.nonzero()[0].tolist())
        pytest.fail(f"{int(bad.sum())} of {bad.numel()} values off, first at {at}: {got[at].item()} for {ref[at].item()}, "
                    f"limit {limit[at].item()}")


def _check_scores(r, ref, tokens, entropy, top):
    if tokens is not None:
        _check(r.logprobs, *ref.logprobs())
    if entropy:
        _check(r.entropy, *ref.entropy())
    if top:
        ids, values, tol = ref.top(top)
        assert bool((r.top_ids == ids).all())
        _check(r.top_logprobs, values, tol)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_scores(kind, cols):
    import paper_2206_10581_amd as tt
    for rows, gap, lead, scale, top, pad in ((1, 0, 0, 1.0, 1, 0.0), (5, 3, 1, 0.7, 64, 0.3), (70, 0, 3, 1.5, 7, 0.5)):
        x, tokens = _logits(cols + rows, (rows, cols), kind, gap, lead), _tokens(rows, rows, cols, pad)
        s = tt.TokenScores(scale)
        ref = Reference(x, tokens, scale)
        _check_scores(s.forward(x, tokens, entropy=True, top=top), ref, tokens, True, top)
        _check_scores(s.forward(x, tokens), ref, tokens, False, 0)
        every = Reference(x, None, scale)
        _check_scores(s.forward(x, top=top), every, None, False, top)
        _check_scores(s.forward(x, entropy=True), every, None, True, 0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out_kind", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_gradient_and_loss(kind, out_kind, cols):
    import torch
    import paper_2206_10581_amd as tt
    for rows, gap, lead, scale, pad in ((1, 0, 0, 1.0, 0.0), (9, 3, 1, 0.7, 0.4), (70, 5, 2, 1.5, 0.3)):
        x, tokens = _logits(cols + rows, (rows, cols), kind, gap, lead), _tokens(rows, rows, cols, pad)
        s = tt.TokenScores(scale)
        ref = Reference(x, tokens, scale)
        g = torch.Generator().manual_seed(rows)
        d, h = torch.randn(rows, generator=g).cuda(), torch.randn(rows, generator=g).cuda()
        r = s.forward(x, tokens, entropy=True, state=True)
        wide = torch.full((rows, cols + gap), 7.0, dtype=getattr(torch, out_kind), device="cuda")
        for dd, dh in ((d, None), (None, h), (d, h)):
            got = s.backward(x, tokens, r.state, dd, dh, out=wide[:, :cols])
            _check(got, *ref.gradient(dd, dh), out_kind)
            assert bool((wide[:, cols:] == 7.0).all())
        every = s.forward(x, entropy=True, state=True)
        _check(s.backward(x, None, every.state, None, h, dtype=getattr(torch, out_kind)),
               *Reference(x, None, scale).gradient(None, h), out_kind)
        for weights in (d, 0.25):
            logprobs, got = s.loss(x, tokens, weights, dtype=getattr(torch, out_kind))
            _check(logprobs, *ref.logprobs())
            _check(got, *ref.gradient(-d if weights is d else torch.full_like(d, -0.25), None), out_kind)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [5, 100, 1000, 20_001])
def test_in_place(kind, cols):
    import torch
    import paper_2206_10581_amd as tt
    x, tokens = _logits(3, (33, cols), kind, 1), _tokens(4, 33, cols, 0.2)
    s, d = tt.TokenScores(), torch.linspace(-1, 1, 33).cuda()
    r = s.forward(x, tokens, entropy=True, state=True)
    want = s.backward(x, tokens, r.state, d, d)
    lost, want_loss = s.loss(x, tokens, d)
    a, b = _logits(3, (33, cols), kind, 1), _logits(3, (33, cols), kind, 1)
    assert s.backward(a, tokens, r.state, d, d, out=a) is a and torch.equal(a, want)
    logprobs, b = s.loss(b, tokens, d, out=b)
    assert torch.equal(b, want_loss) and torch.equal(logprobs, lost)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(3, 4), (2, 200), (40, 1500), (1, 40_000), (5, 40_000), (600, 9000)])
def test_against_differences(kind, rows, cols):
    """Central differences in 64 bits of sum d log p + h entropy, for some logits.  Their own error: a third of the step's square
    times half the third derivative, which is below 0.1 for log p and below 20 for the entropy at these sizes: 4e-8; their
    roundings, 2^-53 of values below 20 over the step, are below 1e-10."""
    import torch
    import paper_2206_10581_amd as tt
    x, tokens = _logits(5, (rows, cols), kind), _tokens(6, rows, cols)
    s = tt.TokenScores(0.8)
    d, h = torch.linspace(-1, 2, rows).cuda(), torch.linspace(1, -1, rows).cuda()
    r = s.forward(x, tokens, entropy=True, state=True)
    got = s.backward(x, tokens, r.state, d, h, dtype=torch.float32).double()
    step = 1e-4
    x64 = x.double()
    tol = Reference(x, tokens, 0.8).gradient(d, h)[1]

    def value(y):
        logp = torch.log_softmax(y * float(np.float32(0.8)), 1)
        return d.double() * logp.gather(1, tokens[:, None])[:, 0] - h.double() * (logp.exp() * logp).sum(1)

    for v in (tokens, (tokens + 1) % cols, x.argmax(1)):
        up = x64.scatter_add(1, v[:, None], torch.full((rows, 1), step, dtype=torch.float64, device="cuda"))
        down = x64.scatter_add(1, v[:, None], torch.full((rows, 1), -step, dtype=torch.float64, device="cuda"))
        slope = (value(up) - value(down)) / (2 * step)
        off = (got.gather(1, v[:, None])[:, 0] - slope).abs() - tol.gather(1, v[:, None])[:, 0] - u * slope.abs()
        assert off.max() < 5e-8


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [3, 47, 200, 1500, 6000, 40_000])
def test_masked_logits(kind, cols):
    """-infinity and the type's lowest value, in some places, everywhere but one, everywhere; at any scale."""
    import torch
    import paper_2206_10581_amd as tt
    low = torch.finfo(getattr(torch, kind)).min
    for scale in (1.0, 30.0, 0.01):
        x, tokens = _logits(7, (8, cols), kind), _tokens(8, 8, cols)
        keep = torch.rand((8, cols), generator=torch.Generator().manual_seed(1)).cuda() < 0.5
        x[0:1] = x[0:1].masked_fill(~keep[0:1], -math.inf)
        x[1:2] = x[1:2].masked_fill(~keep[1:2], low)
        x[2], x[3], x[4], x[5] = -math.inf, low, -math.inf, low
        x[4, cols - 1], x[5, 0], tokens[4], tokens[5] = 2.0, 1.0, cols - 1, 0
        x[6], x[6, cols // 2] = low, -math.inf
        s, ref = tt.TokenScores(scale), Reference(x, tokens, scale)
        ref.logp_tol = ref.logp_tol.nan_to_num(0, 0, 0)
        r = s.forward(x, tokens, entropy=True, top=min(5, cols), state=True)
        assert bool((r.entropy >= 0).all()) and r.logprobs[2] == -math.inf and r.entropy[2] == 0
        assert r.logprobs[4] == 0 and r.logprobs[5] == 0
        _check(r.entropy, *ref.entropy())
        ids, values, tol = ref.top(min(5, cols))
        assert bool((r.top_ids == ids).all())
        fine = values > -3e38                        # what leaves fp32 is -infinity or its lowest values
        _check(torch.where(fine, r.top_logprobs, 0.0), torch.where(fine, values, 0.0), tol)
        assert bool((r.top_logprobs[~fine] < -1e38).all())
        d = torch.linspace(0.5, 1, 8).cuda()
        for dd, dh in ((d, None), (d, d)):
            got = s.backward(x, tokens, r.state, dd, dh, dtype=torch.float32)
            assert bool((got[2] == 0).all())
            _check(got, *ref.gradient(dd, dh))
        logprobs, got = s.loss(x, tokens, -d, dtype=torch.float32)
        assert bool((got[2] == 0).all())
        for v in (logprobs, r.logprobs):
            near = (v > -3e38) | (v == -math.inf)
            want, tol = ref.logprobs()
            _check(torch.where(near, v, 0.0), torch.where(near, torch.where(want < -3.5e38, -math.inf, want), 0.0), tol)
        _check(got, *ref.gradient(d, None))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [9, 300, 3000, 30_000])
def test_nan_and_infinity_stay_in_their_rows(kind, cols):
    import torch
    import paper_2206_10581_amd as tt
    x, tokens = _logits(9, (6, cols), kind), _tokens(10, 6, cols)
    x[1, cols // 2], x[3, cols - 1], x[4, 1], x[4, 3] = math.nan, math.inf, math.nan, math.inf
    x[5], tokens[5] = math.nan, -1                       # left out: not read
    s, d = tt.TokenScores(), torch.ones(6, device="cuda")
    d[5] = math.nan
    r = s.forward(x, tokens, entropy=True, top=3, state=True)
    bad = torch.tensor([False, True, False, True, True, False], device="cuda")
    got, (logprobs, lost) = s.backward(x, tokens, r.state, d, d), s.loss(x, tokens, d)
    for v in (r.logprobs, r.entropy, logprobs):
        assert torch.equal(v.isnan(), bad)
    for g in (got, lost):
        assert torch.equal(g.isnan(), bad[:, None].expand_as(g)) and bool((g[5] == 0).all())
    assert r.top_ids[1, 0] == cols // 2 and r.top_ids[3, 0] == cols - 1 and r.top_ids[4, :2].tolist() == [1, 3]
    assert bool((r.top_ids[5] == -1).all()) and bool((r.top_logprobs[5] == -math.inf).all())
    ok = torch.tensor([0, 2], device="cuda")
    ids, values, tol = Reference(x[ok], tokens[ok], 1.0).top(3)
    assert torch.equal(r.top_ids[ok], ids)


@pytest.mark.parametrize("rows,cols", [(1, 30), (3, 1000), (2, 5000), (1, 100_000), (300, 5000)])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two", "zeros", "blocks"])
def test_likeliest_among_ties_and_orders(rows, cols, order):
    """Lists under attack: every value a new maximum, none, all the same, +0 and -0."""
    import torch
    import paper_2206_10581_amd as tt
    x = torch.arange(cols, dtype=torch.float32).cuda() / cols
    x = {"rising": x, "falling": -x, "equal": x * 0 + 1, "two": (x * cols) % 2, "zeros": torch.where(x * cols % 3 == 0, -0.0, 0.0),
         "blocks": (x * cols // 512)}[order].expand(rows, cols).contiguous()
    tokens = _tokens(1, rows, cols)
    # rising: a rescaling for each value that a thread meets, V / 64 of them at most, each 4 u
    ref = Reference(x, tokens, 1.0, roundings=cols / 64 * 5 + 80)
    s = tt.TokenScores()
    for top in (1, 20, 64):
        _check_scores(s.forward(x, tokens, entropy=True, top=top), ref, tokens, True, top)


def test_repeats_bit_for_bit_and_between_batches():
    import torch
    import paper_2206_10581_amd as tt
    s = tt.TokenScores()
    for rows, cols in ((1, 128_000), (40, 50_257), (700, 4097), (5000, 47)):
        x, tokens = _logits(11, (rows, cols), "bfloat16"), _tokens(12, rows, cols, 0.1)
        a, b = (s.forward(x, tokens, entropy=True, top=5) for _ in range(2))
        assert all(torch.equal(v, w) for v, w in zip(a[:4], b[:4]))
        assert torch.equal(s.loss(x, tokens)[1], s.loss(x, tokens)[1])


def test_no_rows():
    import torch
    import paper_2206_10581_amd as tt
    s = tt.TokenScores()
    x, tokens = torch.empty((0, 50), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    r = s.forward(x, tokens, entropy=True, top=3, state=True)
    assert r.logprobs.shape == (0,) and r.top_ids.shape == (0, 3)
    assert s.backward(x, tokens, r.state, r.logprobs, r.entropy).shape == s.loss(x, tokens)[1].shape == (0, 50)


def test_offsets_beyond_32_bits():
    """2.3e9 logits; rows at the end, and a gradient behind 2^32 bytes."""
    import torch
    import paper_2206_10581_amd as tt
    rows, cols = 18_000, 128_000
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    last = _logits(13, (3, cols), "bfloat16")
    x[-3:] = last
    tokens = torch.full((rows,), -1, device="cuda")
    tokens[-3:] = torch.tensor([5, 127_999, -1], device="cuda")
    tokens[0] = 0
    s = tt.TokenScores()
    r = s.forward(x, tokens, entropy=True, top=3, state=True)
    ref = Reference(last, tokens[-3:], 1.0)
    _check_scores(tt.TokenResult(*(v[-3:] for v in r[:4])), ref, tokens[-3:], True, 3)
    assert abs(r.logprobs[0].item() + math.log(cols)) < 1e-5 and r.top_ids[0].tolist() == [0, 1, 2]
    d = torch.ones(rows, device="cuda")
    g = s.backward(x, tokens, r.state, d, d)
    _check(g[-3:], *ref.gradient(d[:3], d[:3]), "bfloat16")
    assert bool((g[1:-3] == 0).all())
    _, g = s.loss(x, tokens, d, out=x)
    _check(g[-3:], *ref.gradient(-d[:3], None), "bfloat16")


def test_graph_and_streams():
    """Captured calls replayed beside eager ones, on other inputs and on another stream; few rows (parts) and many."""
    import torch
    import paper_2206_10581_amd as tt
    for rows, cols in ((2, 60_000), (300, 1003)):
        s, eager = tt.TokenScores(), tt.TokenScores()
        x, tokens = _logits(14, (rows, cols), "bfloat16"), _tokens(15, rows, cols, 0.2)
        d = torch.linspace(-1, 1, rows).cuda()

        def step(s):
            r = s.forward(x, tokens, entropy=True, top=9, state=True)
            return [*r[:4], s.backward(x, tokens, r.state, d, d), *s.loss(x, tokens, d)]

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step(s)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step(s)
        for k in range(4):
            x.copy_(_logits(16 + k, (rows, cols), "bfloat16"))
            tokens.copy_(_tokens(17 + k, rows, cols, 0.2))
            graph.replay()
            want = step(eager)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    import torch
    import paper_2206_10581_amd as tt
    with pytest.raises(ValueError):
        tt.TokenScores(device="cpu")
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(ValueError):
            tt.TokenScores(scale)
    s, x = tt.TokenScores(), _logits(1, (4, 30), "float32")
    tokens, d = _tokens(1, 4, 30), torch.ones(4, device="cuda")
    state = s.forward(x, tokens, state=True).state
    bad = [lambda: s.forward(x), lambda: s.forward(x, tokens, top=65), lambda: s.forward(x, tokens, top=-1),
           lambda: s.forward(x.t(), tokens), lambda: s.forward(x.cpu(), tokens), lambda: s.forward(x.double(), tokens),
           lambda: s.forward(x[0], tokens), lambda: s.forward(x, tokens.int()), lambda: s.forward(x, tokens[:3]),
           lambda: s.forward(x, tokens.cpu()), lambda: s.forward(x, tokens[:, None]), lambda: s.forward(x[:1].expand(4, 30), tokens),
           lambda: s.backward(x, tokens, state), lambda: s.backward(x, None, state, d), lambda: s.backward(x, tokens, state, d, d),
           lambda: s.backward(x, tokens, state, d.double()), lambda: s.backward(x, tokens, state, d[:3]),
           lambda: s.backward(x[:3], tokens[:3], state, d[:3]), lambda: s.backward(x, tokens, state, d, out=x[:, :29]),
           lambda: s.backward(x, tokens, state, d, out=x, dtype=torch.bfloat16), lambda: s.loss(x, tokens, d.half()),
           lambda: s.loss(x, tokens, d[:3]), lambda: s.loss(x, tokens, torch.ones((), device="cuda"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: s.loss(x, tokens, math.nan), lambda: s.loss(x[:, :29], tokens, out=x[:, 1:]),
                 lambda: s.forward(x[:, :0], tokens)):
        with pytest.raises(tt.TTEmbError):
            call()
