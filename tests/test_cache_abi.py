"""The cache's entry points without a GPU: sizes, and what is refused before
anything is launched."""
import ctypes

import pytest

from paper_2609_00865_amd import mv

FAKE = ctypes.c_void_p(1 << 20)      # aligned, non-null, never dereferenced
ODD = ctypes.c_void_p((1 << 20) + 2)


def status(s):
    return mv.mv_status_string(s).decode()


def shape(layers=2, pages=64, page=16, heads=2, d=128, seqs=8, width=10):
    return mv.CacheShape(layers, pages, page, heads, d, seqs, width)


def cache(**kw):
    return mv.CacheC(*[kw.get(n, FAKE) for n in ("k", "v", "page_table", "seq_len", "page_refs",
                                                "ctl")])


R = ctypes.byref


@pytest.mark.parametrize("bad,want", [(dict(page=24), "MV_ERR_UNSUPPORTED"), (dict(page=8), "MV_ERR_UNSUPPORTED"),
                                      (dict(d=96), "MV_ERR_UNSUPPORTED"), (dict(layers=0), "MV_ERR_SHAPE"),
                                      (dict(pages=-1), "MV_ERR_SHAPE"), (dict(seqs=8193), "MV_ERR_UNSUPPORTED"),
                                      (dict(pages=1 << 27), "MV_ERR_UNSUPPORTED"),
                                      (dict(width=1 << 27), "MV_ERR_UNSUPPORTED"),
                                      (dict(seqs=8192, width=1 << 17), "MV_ERR_UNSUPPORTED")])
def test_shapes(bad, want):
    s, c = shape(**bad), cache()
    assert status(mv.mv_cache_reset(R(s), R(c), None)) == want
    assert status(mv.mv_cache_free(R(s), R(c), 1, FAKE, None)) == want
    assert mv.mv_cache_compact_workspace_bytes(R(s), 1) == 0
    t = mv.TreeAttnShape(1, 1, 4, 0, 0, 0.0)
    assert mv.mv_tree_attn_workspace_bytes(R(s), R(t)) == 0


def test_state_pointers():
    for name in ("k", "v", "page_table", "seq_len", "page_refs", "ctl"):
        for p in (None, ODD):
            c = cache(**{name: p})
            assert status(mv.mv_cache_reset(R(shape()), R(c), None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_reset(R(shape()), None, None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_reset(None, R(cache()), None)) == "MV_ERR_INVALID_ARG"


def test_entries():
    s, c = shape(), cache()
    for n, want in ((-1, "MV_ERR_SHAPE"), (8193, "MV_ERR_UNSUPPORTED"), (0, "MV_OK")):
        assert status(mv.mv_cache_free(R(s), R(c), n, FAKE, None)) == want
        assert status(mv.mv_cache_fork(R(s), R(c), n, FAKE, FAKE, 1, FAKE, 1 << 30, None)) == want
        assert status(mv.mv_cache_compact(R(s), R(c), n, FAKE, FAKE, FAKE, FAKE, 0, FAKE, 1 << 30,
                                          None)) == want
        assert status(mv.mv_cache_reserve(R(s), R(c), n, FAKE, FAKE, 0, FAKE, None, None)) == want
    assert status(mv.mv_cache_reserve(R(s), R(c), 1, None, FAKE, 1, FAKE, None, None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_reserve(R(s), R(c), 1, FAKE, FAKE, -1, FAKE, None, None)) == "MV_ERR_SHAPE"
    assert status(mv.mv_cache_reserve(R(s), R(c), 1, FAKE, FAKE, 1, None, None, None)) == "MV_ERR_INVALID_ARG"
    need = mv.mv_cache_compact_workspace_bytes(R(s), 3)
    assert need > 0
    assert status(mv.mv_cache_fork(R(s), R(c), 3, FAKE, FAKE, 1, FAKE, need - 1, None)) == "MV_ERR_WORKSPACE"
    assert status(mv.mv_cache_fork(R(s), R(c), 3, FAKE, FAKE, 1, None, need, None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_compact(R(s), R(c), 3, FAKE, FAKE, FAKE, None, 2, FAKE, need,
                                      None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_compact(R(s), R(c), 3, FAKE, FAKE, FAKE, FAKE, -2, FAKE, need,
                                      None)) == "MV_ERR_SHAPE"


def spec(rot=128, axes=1, theta=1e6, axis=0):
    return mv.RopeAxesC(rot, axes, theta, (ctypes.c_uint8 * 128)(*([axis] * 128)))


def test_write():
    s, c = shape(), cache()
    w = lambda layer=0, n=3, k=FAKE, ks=256, vs=256, rope=None, pos=None: status(mv.mv_cache_write(
        R(s), R(c), layer, n, FAKE, k, ks, FAKE, vs, R(rope) if rope else None, pos, None))
    assert w(layer=2) == "MV_ERR_SHAPE" and w(layer=-1) == "MV_ERR_SHAPE" and w(n=-1) == "MV_ERR_SHAPE"
    assert w(ks=248) == "MV_ERR_SHAPE" and w(vs=260) == "MV_ERR_SHAPE"
    assert w(k=None) == "MV_ERR_INVALID_ARG" and w(k=ODD) == "MV_ERR_INVALID_ARG"
    assert w(rope=spec(), pos=None) == "MV_ERR_INVALID_ARG"
    assert w(rope=spec(rot=130), pos=FAKE) == "MV_ERR_SHAPE"
    assert w(n=0) == "MV_OK"


def test_rope():
    r = lambda sp, n=2, h=2, d=128, xs=256, os=256, x=FAKE, out=FAKE, pos=FAKE, dr=1: status(
        mv.mv_rope_axes(R(sp), n, h, d, x, xs, pos, dr, out, os, None))
    assert r(spec(rot=3)) == "MV_ERR_SHAPE" and r(spec(rot=0)) == "MV_ERR_SHAPE"
    assert r(spec(rot=130)) == "MV_ERR_SHAPE" and r(spec(axes=9)) == "MV_ERR_SHAPE"
    assert r(spec(axes=0)) == "MV_ERR_SHAPE" and r(spec(axis=1)) == "MV_ERR_SHAPE"
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        assert r(spec(theta=theta)) == "MV_ERR_INVALID_ARG"
    assert r(spec(rot=64), d=100) == "MV_ERR_UNSUPPORTED" and r(spec(), d=264) == "MV_ERR_UNSUPPORTED"
    assert r(spec(), xs=255) == "MV_ERR_SHAPE" and r(spec(), os=250) == "MV_ERR_SHAPE"
    assert r(spec(), dr=0) == "MV_ERR_INVALID_ARG" and r(spec(), pos=None) == "MV_ERR_INVALID_ARG"
    assert r(spec(), x=ODD) == "MV_ERR_INVALID_ARG" and r(spec(), os=264) == "MV_ERR_INVALID_ARG"
    assert r(spec(), n=0) == "MV_OK" and r(spec(), n=-1) == "MV_ERR_SHAPE"
    assert status(mv.mv_rope_axes(None, 2, 2, 128, FAKE, 256, FAKE, 1, FAKE, 256, None)) == "MV_ERR_INVALID_ARG"
    with pytest.raises(ValueError):
        mv.RopeAxes(64, [0] * 33)
    with pytest.raises(ValueError):
        mv.RopeAxes(64, [])
    with pytest.raises(ValueError):
        mv.RopeAxes(64, [8])


def test_tree_attn():
    s, c = shape(), cache()
    t = lambda **kw: mv.TreeAttnShape(*[kw.get(n, v) for n, v in (("B", 2), ("N", 5), ("hq", 4),
                                                                  ("words", 0), ("max_len", 0),
                                                                  ("scale", 0.0))])
    def a(sh, layer=0, ids=FAKE, tree=None, q=FAKE, ws=FAKE, n=1 << 40):
        return status(mv.mv_tree_attn(R(s), R(c), layer, R(sh), ids, FAKE, tree, q, FAKE, FAKE, ws,
                                      n, None))
    need = mv.mv_tree_attn_workspace_bytes(R(s), R(t()))
    assert need > 0
    assert a(t(), n=need - 1) == "MV_ERR_WORKSPACE"
    assert a(t(hq=3)) == "MV_ERR_SHAPE" and a(t(hq=0)) == "MV_ERR_SHAPE" and a(t(B=-1)) == "MV_ERR_SHAPE"
    assert a(t(N=-1)) == "MV_ERR_SHAPE" and a(t(words=-1)) == "MV_ERR_SHAPE"
    assert a(t(max_len=-1)) == "MV_ERR_SHAPE" and a(t(B=8193)) == "MV_ERR_UNSUPPORTED"
    assert a(t(N=1 << 29)) == "MV_ERR_UNSUPPORTED"
    assert a(t(scale=float("nan"))) == "MV_ERR_INVALID_ARG"
    assert a(t(), layer=2) == "MV_ERR_SHAPE" and a(t(), ids=None) == "MV_ERR_INVALID_ARG"
    assert a(t(), tree=FAKE) == "MV_ERR_SHAPE" and a(t(), q=ODD) == "MV_ERR_INVALID_ARG"
    assert a(t(), ws=None) == "MV_ERR_INVALID_ARG"
    assert a(t(B=0)) == "MV_OK" and a(t(N=0)) == "MV_OK"
    m = lambda B=1, N=4, ptr=FAKE, words=1: status(mv.mv_tree_mask(B, N, ptr, FAKE, words, FAKE, None,
                                                                  None))
    assert m(words=0) == "MV_ERR_SHAPE" and m(N=-1) == "MV_ERR_SHAPE" and m(B=-1) == "MV_ERR_SHAPE"
    assert m(ptr=None) == "MV_ERR_INVALID_ARG" and m(N=0) == "MV_OK"


def test_more_pairs_than_a_launch_joins():
    """2^28 pairs of a row and a query head are refused, whichever way they come."""
    for heads, hq, rows in ((64, 64, 1 << 22), (32, 128, 1 << 21), (2, 4, 1 << 26)):
        t = mv.TreeAttnShape(1, rows, hq, 0, 0, 0.0)
        assert mv.mv_tree_attn_workspace_bytes(R(shape(heads=heads)), R(t)) == 0
    t = mv.TreeAttnShape(1, 1 << 20, 64, 0, 0, 0.0)
    assert mv.mv_tree_attn_workspace_bytes(R(shape(heads=64)), R(t)) > 0


def test_workspace_grows_with_the_call():
    """A workspace sized for some rows and entries serves any fewer."""
    s = shape(heads=4)
    last = 0
    for B, N in ((1, 1), (1, 7), (3, 9), (64, 64), (64, 900), (200, 4096)):
        t = mv.TreeAttnShape(B, N, 28, 0, 0, 0.0)
        n = mv.mv_tree_attn_workspace_bytes(R(s), R(t))
        assert n >= last
        last = n
        for m in (1, 100, 5000):
            h = mv.TreeAttnShape(B, N, 28, 0, m, 0.0)
            assert mv.mv_tree_attn_workspace_bytes(R(s), R(h)) <= n
