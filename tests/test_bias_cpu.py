"""Buckets of distances, and the argument checks of the position bias's entry points; nothing is launched."""
from fractions import Fraction

import pytest

from paper_2206_10581_amd import PositionBias
from paper_2206_10581_amd import binding as b


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os
    from paper_2206_10581_amd import build
    if not os.path.exists(build.lib_path()):
        build.build()


def _bucket(n, side, most):
    """The definition in whole numbers: bucket e + k holds n with e (most / e) ** (k / (side - e)) <= n."""
    e = side // 2
    if n < e:
        return n
    return e + max(k for k in range(side - e) if Fraction(n, e) ** (side - e) >= Fraction(most, e) ** k)


@pytest.mark.parametrize("buckets,most", [(32, 128), (4, 2), (4, 3), (8, 20), (64, 1000), (6, 27), (2, 5), (32, 16384 // 4)])
@pytest.mark.parametrize("both", [True, False])
def test_log_buckets(buckets, most, both):
    side = buckets // 2 if both else buckets
    if side < 2 or most <= side // 2:
        with pytest.raises(ValueError):
            PositionBias.log_buckets(buckets, most, both)
        return
    of = PositionBias.log_buckets(buckets, most, both).tolist()
    assert len(of) == 2 * most + 1
    near = [n for n in range(most + 1) if n < 300 or n % 37 == 0 or n > most - 3]
    for n in near:
        assert of[most - n] == _bucket(n, side, most)
        assert of[most + n] == (of[most] if n == 0 else side + _bucket(n, side, most) if both else -1)
    assert of[0] == side - 1


def test_log_buckets_at_exact_powers():
    """16, 32 and 64 start buckets of 32 up to 128, where a logarithm's rounding must not move them."""
    of = PositionBias.log_buckets(32, 128).tolist()
    assert [of[128 - n] for n in (7, 8, 15, 16, 31, 32, 63, 64, 127, 128)] == [7, 8, 9, 10, 11, 12, 13, 14, 15, 15]


def test_log_buckets_refuses():
    for buckets, most, both in ((33, 128, True), (2, 128, True), (1, 128, False), (32, 8, True), (0, 5, False)):
        with pytest.raises(ValueError):
            PositionBias.log_buckets(buckets, most, both)


def _m(data=1 << 20, rows=32, ld=16, cols=16, kind=b.TT_EMB_FP32):
    return b.TTEmbMatrix(data, rows, ld, cols, kind)


def _p(data=1 << 20, batch=2, heads=16, queries=5, keys=7, steps=(560, 35, 7), kind=b.TT_EMB_FP32):
    return b.TTEmbPairs(data, *steps, queries, keys, batch, heads, kind, 0)


def _d(of=256, offsets=0, offset=0, span=128):
    return b.TTEmbDistances(of, offsets, offset, span, 0)


BAD_PAIRS = [_p(data=None), _p(data=258), _p(batch=-1), _p(heads=-1), _p(queries=-1), _p(keys=-1), _p(queries=1 << 30),
             _p(batch=1 << 20, queries=1 << 29, keys=1 << 29), _p(steps=(-1, 35, 7)), _p(steps=(560, -1, 7)), _p(steps=(560, 35, -1)),
             _p(steps=(1 << 41, 35, 7)), _p(kind=3), _p(data=257, kind=b.TT_EMB_FP16), _p(heads=15)]
BAD_DISTANCES = [None, _d(of=0), _d(of=258), _d(offsets=260), _d(span=-1), _d(span=(1 << 20) + 1)]


def test_forward_checks():
    def call(table=_m(), d=_d(), fill=0.0, given=None, out=_p()):
        return b.tt_emb_bias_forward(table, d, fill, given, out, 0)

    for bad in BAD_PAIRS:
        assert call(out=bad) == call(given=bad) == b.TT_EMB_EINVAL
    for bad in BAD_DISTANCES:
        assert call(d=bad) == b.TT_EMB_EINVAL
    for bad in (None, _m(data=None), _m(data=2), _m(ld=15), _m(kind=9), _m(rows=-1), _m(cols=65537, ld=65537)):
        assert call(bad) == b.TT_EMB_EINVAL
    assert call(out=None) == call(fill=float("nan")) == b.TT_EMB_EINVAL
    for other in (_p(batch=3), _p(queries=4), _p(keys=6)):
        assert call(given=other) == b.TT_EMB_EINVAL
    for none in (dict(batch=0), dict(queries=0), dict(keys=0)):
        assert call(out=_p(data=None, **none)) == b.TT_EMB_OK


def test_backward_checks():
    rc, ws = b.tt_emb_bias_workspace_bytes(_p(), 128)
    assert rc == 0 and ws > 0

    def call(g=_p(), d=_d(), out=_m(), at=256, size=ws):
        return b.tt_emb_bias_backward(g, d, out, False, at, size, 0)

    for bad in BAD_PAIRS:
        assert call(bad) == b.TT_EMB_EINVAL
    for bad in BAD_DISTANCES:
        assert call(d=bad) == b.TT_EMB_EINVAL
    for bad in (None, _m(data=None), _m(data=2), _m(ld=15), _m(kind=9), _m(cols=17, ld=17)):
        assert call(out=bad) == b.TT_EMB_EINVAL
    assert call(None) == call(at=0) == call(at=128) == b.TT_EMB_EINVAL
    assert call(size=0) == b.TT_EMB_ENOSPC
    assert call(out=_m(rows=0, data=None)) == b.TT_EMB_OK


def test_workspace_sizes():
    assert b.load_library().tt_emb_bias_workspace_bytes(_p(), 128, None) == b.TT_EMB_EINVAL
    assert b.tt_emb_bias_workspace_bytes(None, 128)[0] == b.tt_emb_bias_workspace_bytes(_p(), -1)[0] == b.TT_EMB_EINVAL
    assert b.tt_emb_bias_workspace_bytes(_p(batch=-1), 128)[0] == b.TT_EMB_EINVAL
    assert b.tt_emb_bias_workspace_bytes(_p(batch=0, data=None), 128) == (0, 0)
    # of a large gradient: a small share of it
    n = b.tt_emb_bias_workspace_bytes(_p(batch=8, queries=2048, keys=2048), 128)[1]
    assert 0 < n < 8 * 16 * 2048 * 2048 // 32
