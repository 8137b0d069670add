"""The calls of decoding over a shared and a bounded cache refuse bad arguments on the host (nothing is launched), and the 64-bit
models that their GPU tests use are pinned.  CPU only."""
import numpy as np
import pytest

from oracle import handoff_oracle as H
from test_handoff_args import F, cache, heads, mb  # noqa: F401  (mb: the fixture)

BAD_CACHES = (("E", dict(pool=0)), ("E", dict(pool=F + 8)), ("E", dict(table=0)), ("E", dict(length=0)), ("E", dict(refs=0)),
              ("E", dict(status=0)), ("E", dict(typ=2)), ("E", dict(layers=0)), ("E", dict(pages=0)), ("E", dict(max_pages=0)),
              ("U", dict(dh=60)), ("U", dict(dh=264)), ("U", dict(page=1025)), ("U", dict(seqs=262145)), ("U", dict(max_pages=1 << 27)))


def shared(mb, c, layer=0, q=None, seqs=F, n=2, starts=F, groups=1, scale=1.0, out=None, ws=F):  # noqa: F811
    h = heads(mb, n=2, row=128)
    return mb.lib.map_cache_attend_shared(c, layer, h if q is None else q, seqs, n, starts, groups, scale,
                                          h if out is None else out, ws, None)


def weigh(mb, c, layer=0, q=None, seqs=F, n=2, scale=1.0, out=None, weights=F, ws=F):  # noqa: F811
    h = heads(mb, n=2, row=128)
    return mb.lib.map_cache_attend_weigh(c, layer, h if q is None else q, seqs, n, scale, h if out is None else out, weights, ws, None)


def both(mb, c, **bad):  # noqa: F811
    """What the two attentions answer to the same bad arguments."""
    return shared(mb, c, **bad), weigh(mb, c, **bad)


def test_attend_refusals(mb):  # noqa: F811
    code, c = {"E": mb.MAP_EINVAL, "U": mb.MAP_EUNSUPPORTED}, cache(mb)
    for kind, bad in BAD_CACHES:
        b = cache(mb, **bad)
        assert both(mb, b) == (code[kind],) * 2, bad
        assert mb.lib.map_cache_attend_shared_workspace(b, 4, 4, 2) == 0
        assert mb.lib.map_cache_attend_weigh_workspace(b, 4, 4) == 0
    h = heads(mb, n=2, row=128)
    for bad in (dict(layer=2), dict(layer=-1), dict(q=heads(mb, n=3)), dict(q=heads(mb, n=4)), dict(out=heads(mb, n=4)), dict(n=-1),
                dict(seqs=None), dict(ws=None), dict(ws=F + 8), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(q=heads(mb, p=0, n=2)), dict(q=heads(mb, p=F + 8, n=2)), dict(q=heads(mb, row=-8, n=2)),
                dict(q=heads(mb, row=132, n=2)), dict(out=heads(mb, row=127, n=2)), dict(out=heads(mb, row=120, n=2)),
                dict(out=heads(mb, row=0, n=2))):
        assert both(mb, c, **bad) == (mb.MAP_EINVAL,) * 2, bad
    for bad in (dict(n=65536, out=h, q=h),):
        assert both(mb, c, **bad) == (mb.MAP_EUNSUPPORTED,) * 2
    for dh in (8, 40, 72, 112, 160, 248):
        assert both(mb, cache(mb, dh=dh), q=heads(mb, n=2, row=512, head=256), out=heads(mb, n=2, row=512, head=256)) == \
            (mb.MAP_EUNSUPPORTED,) * 2
    # each call's own arguments
    assert shared(mb, c, starts=None) == shared(mb, c, groups=0) == shared(mb, c, groups=-1) == mb.MAP_EINVAL
    assert shared(mb, c, groups=65536) == mb.MAP_EUNSUPPORTED
    assert weigh(mb, c, weights=None) == weigh(mb, c, weights=F + 2) == mb.MAP_EINVAL
    assert shared(mb, c, n=0, seqs=None, ws=None, starts=None) == weigh(mb, c, n=0, seqs=None, ws=None, weights=None) == mb.MAP_OK
    # scores of more than 2^46 bytes; 2^31 rows of queries
    wide, many = cache(mb, max_pages=(1 << 27) - 1), mb._pack_heads(F, 65534 * 64, 64, 65534)
    assert weigh(mb, wide, q=many, out=many, n=65535) == mb.MAP_EUNSUPPORTED
    assert mb.lib.map_cache_attend_weigh_workspace(wide, 65534, 65535) == 0
    assert shared(mb, c, q=many, out=many, n=65535) == shared(mb, c, q=many, out=many, n=32770) == mb.MAP_EUNSUPPORTED
    assert mb.lib.map_cache_attend_shared_workspace(c, 65534, 32770, 1) == 0 < mb.lib.map_cache_attend_shared_workspace(c, 65534, 32769, 1)
    for bad in ((0, 4, 1), (65536, 4, 1), (4, -1, 1), (4, 65536, 1), (4, 4, 0), (4, 4, 65536)):
        assert mb.lib.map_cache_attend_shared_workspace(c, *bad) == 0, bad
        if bad[2] == 1:
            assert mb.lib.map_cache_attend_weigh_workspace(c, *bad[:2]) == 0, bad
    # a score of each row that a sequence can have (4 pages of 16), a result of each head in fp32 twice
    assert mb.lib.map_cache_attend_weigh_workspace(c, 4, 3) >= 4 * 3 * 64 * 4
    assert mb.lib.map_cache_attend_shared_workspace(c, 4, 3, 2) >= 2 * 4 * 3 * 64 * 4


def test_evict_refusals(mb):  # noqa: F811
    lib, E, U = mb.lib, mb.MAP_EINVAL, mb.MAP_EUNSUPPORTED
    for kind, bad in BAD_CACHES:
        b = cache(mb, **bad)
        assert lib.map_cache_evict(b, F, F, 1, F, F, 1, F, None) == {"E": E, "U": U}[kind], bad
        assert lib.map_cache_evict_workspace(b, 1, 1) == 0
    c = cache(mb)
    for args in ((None, F, 1, F, F, 1, F), (F + 2, F, 1, F, F, 1, F), (F, None, 1, F, F, 1, F), (F, F, -1, F, F, 1, F),
                 (F, F, 1, F, F, -1, F), (F, F, 1, F, F, 1, None), (F, F, 1, F, F, 1, F + 8)):
        assert lib.map_cache_evict(c, *args, None) == E, args
    assert lib.map_cache_evict(c, F, F, 4097, F, F, 1, F, None) == U
    many = cache(mb, page=1, max_pages=1 << 20)
    assert lib.map_cache_evict(many, F, F, 2048, F, F, 1, F, None) == U and lib.map_cache_evict_workspace(many, 2048, 1) == 0
    heads_of_all = cache(mb, hk=8, layers=1024)                       # 4096 * 8192 units
    assert lib.map_cache_evict(heads_of_all, F, F, 4096, F, F, 1, F, None) == U and lib.map_cache_evict_workspace(heads_of_all, 4096, 1) == 0
    assert lib.map_cache_evict_workspace(heads_of_all, 2048, 1) > 0 == lib.map_cache_evict_workspace(heads_of_all, 2048, -1)
    assert lib.map_cache_evict_workspace(many, 2047, 1) >= 2047 * 4 << 20
    assert lib.map_cache_evict(c, None, None, 0, None, None, 0, None, None) == mb.MAP_OK


def test_eviction_model_by_hand():
    m = H.Pages(6, 4, 3, 3)
    m.extend([0, 1], [7, 3], 10)                                     # sequence 0: pages 0 and 1, sequence 1: page 2
    assert m.fork([0], [2]) == [(12, 4), (13, 5), (14, 6)]           # page 0 shared, page 3 its own
    w = np.zeros((1, 3, 1, 12), np.float32)
    w[0, 0, 0, :7] = [9, 1, 5, 0, 5, 2, 7]
    # of rows 1 .. 5 two stay: 5 and 5; row 0 stays in front of them, row 6 behind; page 0 is the fork's too.  Of sequence 1's
    # three rows of weight 0 the first two stay where they are.
    assert m.evict([-1, 0, 1], [0, 1, 0], [0, 1, 0], 2, w) == [(0, 0, [16, 17, 18, 19], [0, 2, 4, 6]), (0, 0, [], [])]
    assert m.table == [[4], [2], [0, 3]] and m.length == [4, 2, 7] and m.refs == [1, 0, 1, 1, 1, 0]
    assert w[0, 0, 0].tolist() == [9, 5, 5, 7] + [0] * 8
    # a tie goes to the row in front, NaN before all, k = 0 leaves nothing of the window
    w[0, 2, 0, :7] = [1, np.nan, 1, 3, 1, -1, 0]
    assert m.evict([2], [0], [0], 3, w) == [(0, 0, [2], [3])]
    assert np.isnan(w[0, 2, 0, 1]) and w[0, 2, 0, [0, 2, 3]].tolist() == [1, 3, 0] and m.table[2] == [0]
    assert m.evict([2], [1], [1], 0, w) == [(0, 0, [1], [2])] and m.length[2] == 2
    # refused: the same twice, a window that begins before the sequence, too few pages
    before = (list(m.length), list(m.refs))
    assert m.evict([2, 2], [0, 0], [0, 0], 1, w) is None and m.evict([2], [-1], [0], 1, w) is None
    assert m.evict([3], [0], [0], 1, w) is None and (m.length, m.refs) == before


def test_weights_model():
    q, k = np.array([[1.0, 0.0], [0.0, 1.0]]), np.zeros((2, 1, 2))
    k[1, 0, 0] = np.log(3.0)
    assert np.allclose(H.attend_weights(q, k, 1.0), [[0.25 + 0.5, 0.75 + 0.5]])
