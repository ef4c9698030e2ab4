"""Argument checks of the plain-table, norm and clipping entry points; nothing is launched."""
import ctypes

import pytest

from paper_2206_10581_amd import binding as b


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os
    from paper_2206_10581_amd import build
    if not os.path.exists(build.lib_path()):
        build.build()


def _m(data=256, rows=10, ld=16, cols=16, kind=b.TT_EMB_FP32):
    return b.TTEmbMatrix(data, rows, ld, cols, kind)


BAD = [_m(data=None), _m(data=258), _m(rows=-1), _m(ld=15), _m(cols=0), _m(cols=65537, ld=65537), _m(kind=3), _m(kind=-1),
       _m(rows=1 << 31), _m(data=257, kind=b.TT_EMB_BF16), _m(ld=1 << 41)]


def test_dense_forward_checks():
    good = _m()
    for bad in BAD:
        assert b.tt_emb_dense_forward(bad, 256, 1.0, good, 0) == b.TT_EMB_EINVAL
        assert b.tt_emb_dense_forward(good, 256, 1.0, bad, 0) == b.TT_EMB_EINVAL
    assert b.tt_emb_dense_forward(good, 0, 1.0, good, 0) == b.TT_EMB_EINVAL
    assert b.tt_emb_dense_forward(good, 260, 1.0, good, 0) == b.TT_EMB_EINVAL
    assert b.tt_emb_dense_forward(good, 256, 1.0, _m(cols=8), 0) == b.TT_EMB_EINVAL
    assert b.tt_emb_dense_forward(good, 256, 1.0, _m(rows=1 << 30), 0) == b.TT_EMB_EINVAL
    assert b.tt_emb_dense_forward(good, 0, 1.0, _m(data=None, rows=0), 0) == b.TT_EMB_OK     # no ids, no rows
    lib = b.load_library()
    assert lib.tt_emb_dense_forward(None, 256, 1.0, ctypes.byref(good), None) == b.TT_EMB_EINVAL
    assert lib.tt_emb_dense_forward(ctypes.byref(good), 256, 1.0, None, None) == b.TT_EMB_EINVAL


def test_dense_workspace():
    assert b.load_library().tt_emb_dense_workspace_bytes(16, 8, None) == b.TT_EMB_EINVAL
    for cols, batch in ((0, 8), (65537, 8), (16, 0), (16, 1 << 30)):
        assert b.tt_emb_dense_workspace_bytes(cols, batch)[0] == b.TT_EMB_EINVAL
    sizes = [b.tt_emb_dense_workspace_bytes(cols, batch) for cols in (1, 100, 4096)
             for batch in (1, 33, 10_000, 131_072, 131_073, 300_000, 600_000, 2_000_000)]
    assert all(rc == 0 and n % 256 == 0 for rc, n in sizes)
    for k in range(0, len(sizes), 8):
        assert [n for _, n in sizes[k:k + 8]] == sorted(n for _, n in sizes[k:k + 8])   # a workspace fits all smaller batches


@pytest.mark.parametrize("cols", [1, 63, 512, 4096, 65536])
def test_a_workspace_fits_every_smaller_batch(cols):
    """Tiles of sorted positions get larger where batches do: the smaller ones must not need more."""
    pieces = (cols + 7) // 8
    turn = [min(65535, (64 << 16) // pieces), 65536, (64 << 16) // pieces]
    batches = sorted({max(1, n + d) for n in (1, 8, 100, *turn) for d in (-1, 0, 1)} | {2 * n for n in turn})
    need = [b.tt_emb_dense_workspace_bytes(cols, n) for n in batches if n < 1 << 30]
    assert all(rc == 0 for rc, _ in need)
    assert [n for _, n in need] == sorted(n for _, n in need)


def test_dense_backward_checks():
    good, ws = _m(), b.tt_emb_dense_workspace_bytes(16, 10)[1]

    def call(ids=256, grad=good, out=good, at=256, size=ws):
        return b.tt_emb_dense_backward(ids, grad, 1.0, -1, out, False, at, size, 0)

    for bad in BAD:
        assert call(grad=bad) == b.TT_EMB_EINVAL and call(out=bad) == b.TT_EMB_EINVAL
    assert call(ids=0) == call(ids=260) == call(out=_m(cols=8)) == call(at=0) == call(at=255) == b.TT_EMB_EINVAL
    assert call(size=ws - 1) == b.TT_EMB_ENOSPC
    assert call(out=_m(rows=0, data=None)) == b.TT_EMB_OK          # a table without rows has no gradient


def test_norm_and_clip_checks():
    rc, ws = b.tt_emb_norm_workspace_bytes(2)
    assert rc == 0 and b.tt_emb_norm_workspace_bytes(-1)[0] == b.TT_EMB_EINVAL
    assert b.load_library().tt_emb_norm_workspace_bytes(2, None) == b.TT_EMB_EINVAL
    assert b.tt_emb_norm_workspace_bytes(1000)[1] > ws

    def values(*second):
        return (b.TTEmbValues * 2)(b.TTEmbValues(256, 8, b.TT_EMB_FP32, 0), b.TTEmbValues(*second, 0))

    good = values(512, 8, b.TT_EMB_BF16)
    bad = [values(None, 8, 0), values(514, 8, 0), values(513, 8, 1), values(512, -1, 0), values(512, (1 << 40) + 1, 0),
           values(512, 8, 3)]

    def norm(v=good, n=2, scale=1.0, out=256, at=256, size=ws):
        return b.tt_emb_grad_norm(v, n, scale, out, at, size, 0)

    def clip(v=good, out=None, scale=1.0, limit=1.0, eps=0.0, norm=256, at=256, size=ws):
        return b.tt_emb_grad_clip(v, out, 2, scale, limit, eps, norm, at, size, 0)

    for v in bad:
        assert norm(v) == clip(v) == clip(out=v) == b.TT_EMB_EINVAL
    nan = float("nan")
    assert norm(n=-1) == norm(v=None) == norm(scale=nan) == norm(out=0) == norm(out=258) == b.TT_EMB_EINVAL
    assert norm(at=0) == norm(at=128) == clip(limit=-1.0) == clip(limit=nan) == clip(eps=nan) == b.TT_EMB_EINVAL
    assert clip(eps=-1.0) == clip(out=values(512, 9, 1)) == clip(scale=nan) == b.TT_EMB_EINVAL
    assert norm(size=ws - 1) == clip(size=ws - 1) == b.TT_EMB_ENOSPC
