"""Log probabilities of masked tokens, and lists that one wavefront makes, against 64 bits.  A reference of -infinity or NaN has
to be met as it is; the tolerances of the others are those of test_tokens."""
import math

import pytest
from test_tokens import TYPES, Reference, _logits, _tokens, u

pytestmark = pytest.mark.gpu


def _same(got, ref, tol):
    import torch
    got, finite = got.double(), ref.isfinite()
    limit = torch.where(finite, tol + u * ref.abs(), 0.0)
    good = torch.where(finite, (got - ref).abs() <= limit, (got == ref) | (got.isnan() & ref.isnan()))
    if not bool(good.all()):
        at = tuple((~good).nonzero()[0].tolist())
        pytest.fail(f"{int((~good).sum())} of {good.numel()} values off, first at {at}: {got[at].item()} for {ref[at].item()}, "
                    f"limit {limit[at].item()}")


def _same_lists(r, ref, top):
    ids, values, tol = ref.top(top)
    assert bool((r.top_ids == ids).all())
    _same(r.top_logprobs, values, tol)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(9, 3), (9, 47), (9, 200), (70, 300), (600, 1003), (9, 1500), (9, 6000), (3, 40_000), (200, 40_000)])
def test_masked_tokens_have_no_probability(kind, rows, cols):
    """Half of the logits are -infinity, half of the tokens among them; of the last two rows all, and all but the token."""
    import torch
    import paper_2206_10581_amd as tt
    x, tokens = _logits(1, (rows, cols), kind, 1), _tokens(2, rows, cols, 0.1)
    keep = torch.rand((rows, cols), generator=torch.Generator().manual_seed(3)).cuda() < 0.5
    x.masked_fill_(~keep, -math.inf)
    x[-2:] = -math.inf
    tokens[-2:] = torch.tensor([cols - 1, cols // 2])
    x[-1, cols // 2] = -2.0
    ref = Reference(x, tokens, 0.8)
    want, tol = ref.logprobs()
    assert want[-1] == 0 and (rows < 60 or bool((want[:-2] == -math.inf).any()) and bool((want[:-2] < -0.1).isfinite().any()))
    s = tt.TokenScores(0.8)
    for top in (0, 1, 20, 64):                                # with few columns: places that nothing fills
        r = s.forward(x, tokens, entropy=True, top=top)
        _same(r.logprobs, want, tol)
        _same(r.entropy, *ref.entropy())
        if top:
            _same_lists(r, ref, top)
    logprobs, _ = s.loss(x, tokens)
    _same(logprobs, want, tol)


@pytest.mark.parametrize("rows,cols,kind", [(600, 1003, "float32"), (600, 4097, "float32"), (600, 2500, "bfloat16"), (600, 8000, "float16"),
                                            (600, 100, "bfloat16"), (600, 4, "float32")])
@pytest.mark.parametrize("order", ["random", "rising", "falling", "equal", "two", "few", "nan"])
def test_lists_of_a_wavefront(rows, cols, kind, order):
    """Blocks of 64 threads: many rows of up to 1024 pieces, and long lists of narrow rows."""
    import torch
    import paper_2206_10581_amd as tt
    line = torch.arange(cols, dtype=torch.float32).cuda() / cols
    if order in ("rising", "falling", "equal", "two"):
        x = {"rising": line, "falling": -line, "equal": line * 0 + 1, "two": line * cols % 2}[order]
        x = x.expand(rows, cols).to(getattr(torch, kind)).contiguous()
    else:
        x = _logits(4, (rows, cols), kind)
    if order == "few":                                        # a handful that are allowed, at other places in every row
        g = torch.Generator().manual_seed(5)
        keep = torch.zeros((rows, cols), dtype=torch.bool).scatter_(1, torch.randint(0, cols, (rows, 5), generator=g), True).cuda()
        x.masked_fill_(~keep, -math.inf)
    tokens = _tokens(6, rows, cols, 0.1)
    ref = Reference(x, tokens, 1.0, roundings=cols / 64 * 5 + 80)
    if order == "nan":
        x[3, cols // 3], x[3, cols - 1], x[5] = math.nan, math.nan, math.nan
        tokens[3], tokens[5] = 0, 1
        ref = Reference(x, tokens, 1.0)
    s = tt.TokenScores()
    for top in (1, 20, 64):
        r = s.forward(x, tokens, top=top)
        if order != "nan":
            _same(r.logprobs, *ref.logprobs())
            _same_lists(r, ref, top)
            continue
        first = sorted({cols // 3, cols - 1})
        assert top == 1 or r.top_ids[3, :2].tolist() == first
        assert r.top_ids[3, 0] == first[0] and r.top_ids[5].tolist() == [k if k < cols else -1 for k in range(top)]
        for row in (3, 5):
            assert r.logprobs[row].isnan() and bool(r.top_logprobs[row, :min(top, cols)].isnan().all())
        ok = torch.ones(rows, dtype=torch.bool, device="cuda")
        ok[3] = ok[5] = False
        _same_lists(tt.TokenResult(None, None, r.top_ids[ok], r.top_logprobs[ok]), Reference(x[ok], tokens[ok], 1.0), top)
