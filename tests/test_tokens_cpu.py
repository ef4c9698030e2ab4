"""Argument checks of the entry points for scores of logits; nothing is launched."""
import ctypes

import pytest

from paper_2206_10581_amd import binding as b


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os
    from paper_2206_10581_amd import build
    if not os.path.exists(build.lib_path()):
        build.build()


def _m(data=1 << 20, rows=10, ld=16, cols=16, kind=b.TT_EMB_FP32):
    return b.TTEmbMatrix(data, rows, ld, cols, kind)


def _out(logprob=256, entropy=0, state=0, top_ids=0, top_logprob=0, top=0):
    return b.TTEmbTokenOut(logprob, entropy, state, top_ids, top_logprob, top, 0)


BAD = [None, _m(data=None), _m(data=258), _m(rows=-1), _m(ld=15), _m(cols=0), _m(cols=(1 << 30) + 1, ld=1 << 31), _m(kind=3),
       _m(kind=-1), _m(rows=1 << 30), _m(data=257, kind=b.TT_EMB_BF16), _m(ld=(1 << 40) + 1)]
SCALES = [0.0, -1.0, float("nan"), float("inf"), 2e38]
WS = 1 << 20


def test_workspace():
    rc, n = b.tt_emb_token_workspace_bytes()
    assert rc == 0 and 0 < n < WS
    assert b.load_library().tt_emb_token_workspace_bytes(None) == b.TT_EMB_EINVAL


def test_scores_checks():
    def call(m=_m(), tokens=256, scale=1.0, out=_out(), at=256, size=WS):
        return b.tt_emb_token_scores(m, tokens, scale, out, at, size, 0)

    for bad in BAD:
        assert call(bad) == b.TT_EMB_EINVAL
    for scale in SCALES:
        assert call(scale=scale) == b.TT_EMB_EINVAL
    assert call(out=None) == call(tokens=260) == call(at=0) == call(at=255) == b.TT_EMB_EINVAL
    assert call(out=_out(0)) == b.TT_EMB_EINVAL                         # nothing wanted
    assert call(tokens=0) == b.TT_EMB_EINVAL                            # log probabilities of no token
    assert call(out=_out(258)) == call(out=_out(entropy=2)) == call(out=_out(state=1)) == b.TT_EMB_EINVAL
    for ids, values, top in ((256, 0, 1), (0, 256, 1), (256, 256, 0), (256, 256, 65), (260, 256, 1), (256, 258, 1)):
        assert call(out=_out(256, 0, 0, ids, values, top)) == b.TT_EMB_EINVAL
    assert call(size=b.tt_emb_token_workspace_bytes()[1] - 1) == b.TT_EMB_ENOSPC
    assert call(_m(rows=0, data=None), tokens=0, out=_out(0)) == b.TT_EMB_OK


def test_backward_checks():
    def call(m=_m(), tokens=256, scale=1.0, state=256, entropy=256, d=256, h=256, dx=_m(data=2 << 20)):
        return b.tt_emb_token_backward(m, tokens, scale, state, entropy, d, h, dx, 0)

    for bad in BAD:
        assert call(bad) == call(dx=bad) == b.TT_EMB_EINVAL
    for scale in SCALES:
        assert call(scale=scale) == b.TT_EMB_EINVAL
    assert call(state=0) == call(entropy=0) == call(d=0, h=0) == call(tokens=0) == call(tokens=260) == b.TT_EMB_EINVAL
    assert call(state=258) == call(entropy=258) == call(d=258) == call(h=258) == b.TT_EMB_EINVAL
    assert call(dx=_m(2 << 20, rows=9)) == call(dx=_m(2 << 20, cols=15)) == b.TT_EMB_EINVAL
    assert call(_m(rows=0, data=None), 0, 1.0, 0, 0, 0, 0, _m(rows=0, data=None)) == b.TT_EMB_OK


def test_a_gradient_is_written_over_its_logits_or_apart_from_them():
    at = 1 << 20

    def call(m, dx):                                                   # no state: refused later than for an overlap
        return b.load_library().tt_emb_token_loss(ctypes.byref(m), 256, 1.0, None, 1.0, 256, ctypes.byref(dx), 256, 0, None)

    ok, refused = b.TT_EMB_ENOSPC, b.TT_EMB_EINVAL
    assert call(_m(at), _m(at)) == ok
    assert call(_m(at), _m(at, kind=b.TT_EMB_BF16)) == refused
    assert call(_m(at), _m(at, ld=17)) == refused
    assert call(_m(at, rows=1), _m(at, rows=1, ld=17)) == ok
    size = 4 * (9 * 16 + 16)
    assert call(_m(at), _m(at + size)) == call(_m(at + size), _m(at)) == ok
    assert call(_m(at), _m(at + size - 4)) == call(_m(at + size - 4), _m(at)) == call(_m(at), _m(at + 4)) == refused
    # columns of one wider buffer
    assert call(_m(at, ld=32), _m(at + 64, ld=32)) == call(_m(at + 64, ld=32), _m(at, ld=32)) == ok
    assert call(_m(at, ld=32), _m(at + 60, ld=32)) == call(_m(at + 68, ld=32), _m(at, ld=32)) == refused
    assert call(_m(at, ld=32), _m(at + 64, ld=64, kind=b.TT_EMB_BF16)) == ok


def test_loss_checks():
    def call(m=_m(), tokens=256, scale=1.0, weights=0, weight=1.0, logprob=256, dx=_m(data=2 << 20), at=256, size=WS):
        return b.tt_emb_token_loss(m, tokens, scale, weights, weight, logprob, dx, at, size, 0)

    for bad in BAD:
        assert call(bad) == call(dx=bad) == b.TT_EMB_EINVAL
    for scale in SCALES:
        assert call(scale=scale) == b.TT_EMB_EINVAL
    assert call(tokens=0) == call(logprob=0) == call(weights=2) == call(logprob=2) == b.TT_EMB_EINVAL
    assert call(weight=float("nan")) == call(weight=float("inf")) == call(at=0) == call(at=64) == b.TT_EMB_EINVAL
    assert call(size=0) == b.TT_EMB_ENOSPC
    assert call(_m(rows=0, data=None), tokens=0, logprob=0, dx=_m(rows=0, data=None)) == b.TT_EMB_OK
