"""Scores that a bias is added to and an output that shares some of their memory: refused before anything is launched."""
import pytest

from paper_2206_10581_amd import binding as b

AT = 1 << 20
SIZES = (2, 3, 5, 7)                                           # batch, heads, queries, keys
DENSE = (105, 35, 7)


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os
    from paper_2206_10581_amd import build
    if not os.path.exists(build.lib_path()):
        build.build()


def _p(data=AT, steps=DENSE, kind=b.TT_EMB_FP32, sizes=SIZES):
    batch, heads, queries, keys = sizes
    return b.TTEmbPairs(data, *steps, queries, keys, batch, heads, kind, 0)


def _call(given, out):
    table = b.TTEmbMatrix(256, 4, out.heads, out.heads, b.TT_EMB_FP32)
    return b.tt_emb_bias_forward(table, b.TTEmbDistances(256, 0, 0, 3, 0), 0.0, given, out, 0)


WIDE = (5 * 3 * 20, 20, 3 * 20)                                # queries before heads, and 20 places a row


@pytest.mark.parametrize("given,out", [
    (_p(AT + 4), _p()), (_p(), _p(AT + 4)),                    # a place further
    (_p(), _p(AT + 4 * 7)), (_p(), _p(AT + 4 * 35)),           # a row, a head further
    (_p(), _p(AT + 4 * (210 - 1))), (_p(AT + 4 * (210 - 1)), _p()),    # the last place
    (_p(), _p(kind=b.TT_EMB_BF16)), (_p(kind=b.TT_EMB_BF16), _p(kind=b.TT_EMB_FP16)),
    (_p(AT + 2, kind=b.TT_EMB_BF16), _p(kind=b.TT_EMB_FP16)),
    (_p(), _p(steps=(105, 7, 21))), (_p(), _p(AT + 400, steps=(0, 35, 7))),
    (_p(steps=(0, 35, 7)), _p()), (_p(AT + 4 * 105, steps=(0, 35, 7)), _p()),
    (_p(steps=WIDE), _p(AT + 4 * 6, steps=WIDE)), (_p(AT + 4 * 6, steps=WIDE), _p(steps=WIDE)),
    (_p(steps=WIDE), _p(AT + 4 * 15, steps=WIDE)),             # the next head's row
    (_p(steps=WIDE), _p(AT + 4 * (300 + 60 - 20 - 6), steps=WIDE)),
    (_p(sizes=(1, 1, 1, 7)), _p(AT + 24, sizes=(1, 1, 1, 7), steps=(1, 2, 3))),
])
def test_refused(given, out):
    assert _call(given, out) == b.TT_EMB_EINVAL
