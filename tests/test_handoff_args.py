"""The hand-off's calls refuse bad arguments on the host (nothing is launched), and the 64-bit models that its GPU
tests use are pinned.  CPU only."""
import ctypes
import math

import numpy as np
import pytest

from oracle import handoff_oracle as H

F = 256            # a non-null, aligned stand-in; nothing is dereferenced or launched on an argument error


@pytest.fixture(scope="module")
def mb():
    from paper_2608_06411_gb300 import build_lib
    build_lib.build()
    from paper_2608_06411_gb300 import binding
    return binding


def heads(mb, p=F, row=256, head=64, n=4):
    return mb._pack_heads(p, row, head, n)


def cache(mb, pool=F, table=F, length=F, refs=F, status=F, typ=0, layers=2, pages=8, hk=2, page=16, dh=64, seqs=4,
          max_pages=4):
    return mb._pack_cache(pool, table, length, refs, status, typ, layers, pages, hk, page, dh, seqs, max_pages)


@pytest.fixture(scope="module")
def rope(mb):
    return mb.Rope(64, [1.0 / (i + 1) for i in range(32)], axis=[i % 3 for i in range(32)])


def test_rope_plan_refusals(mb):
    for bad in (dict(dh=0), dict(dh=257), dict(inv_freq=[1.0] * 40), dict(inv_freq=[math.inf]), dict(inv_freq=[math.nan]),
                dict(axis=[2], inv_freq=[1.0], n_axes=2), dict(axis=[-1], inv_freq=[1.0], n_axes=2), dict(n_axes=0),
                dict(n_axes=5), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)):
        with pytest.raises(mb.MapError) as e:
            mb.Rope(**{**dict(dh=64, inv_freq=[1.0, 0.5]), **bad})
        assert e.value.code == mb.MAP_EINVAL
    with pytest.raises(ValueError):
        mb.Rope(64, [1.0, 0.5], axis=[0])
    assert mb.lib.map_rope_init(64, 64, 0, 1, None, None, 0.0, ctypes.byref(ctypes.c_void_p())) == mb.MAP_EINVAL
    assert mb.lib.map_rope_init(64, 0, 0, 1, None, None, 0.0, None) == mb.MAP_EINVAL
    mb.Rope(64, []).close()
    mb.lib.map_rope_destroy(None)
    assert mb.lib.map_qk_rotate_grad_workspace(None) == 0


def test_rotate_refusals(mb, rope):
    L, E, h = mb.lib.map_qk_rotate, mb.MAP_EINVAL, heads(mb)
    assert L(None, 0, 4, F, h, h, None, None, h, h, None) == E
    assert L(rope.h, 3, 4, F, h, h, None, None, h, h, None) == E
    assert L(rope.h, 0, -1, F, h, h, None, None, h, h, None) == E
    assert L(rope.h, 0, 4, None, h, h, None, None, h, h, None) == E
    assert L(rope.h, 0, 4, F, None, None, None, None, None, None, None) == E
    assert L(rope.h, 0, 4, F, h, None, None, None, None, None, None) == E                       # no output
    assert L(rope.h, 0, 4, F, h, h, None, None, h, heads(mb, n=2), None) == E                   # fewer heads out
    assert L(rope.h, 0, 4, F, heads(mb, row=-1), None, None, None, h, None, None) == E
    assert L(rope.h, 0, 4, F, heads(mb, p=F + 1), None, None, None, h, None, None) == E         # half an element off
    assert L(rope.h, 2, 4, F, heads(mb, p=F + 2), None, None, None, h, None, None) == E
    for o in (heads(mb, head=63), heads(mb, row=0), heads(mb, row=255), heads(mb, head=0)):     # overlapping outputs
        assert L(rope.h, 0, 4, F, h, None, None, None, o, None, None) == E
    assert L(rope.h, 0, 1 << 30, F, h, None, None, None, h, None, None) == E                    # rows * heads
    assert L(rope.h, 0, 0, F, h, h, None, None, h, h, None) == mb.MAP_OK
    assert L(rope.h, 0, 0, None, h, h, None, None, h, h, None) == mb.MAP_OK


def test_rotate_grad_refusals(mb, rope):
    L, E, h = mb.lib.map_qk_rotate_grad, mb.MAP_EINVAL, heads(mb)

    def call(typ=0, rows=4, pos=F, g=h, x=h, w=F, dx=h, dw=F, ws=F):
        return L(rope.h, typ, rows, pos, g, None, x, None, w, None, dx, None, dw, None, ws, None)

    for bad in (dict(typ=9), dict(rows=-1), dict(pos=None), dict(g=None), dict(x=None), dict(x=heads(mb, n=2)), dict(dx=None),
                dict(dx=heads(mb, head=8)), dict(dw=None), dict(ws=None), dict(ws=F + 4)):
        assert call(**bad) == E, bad


def test_cache_refusals(mb, rope):
    lib, E, U = mb.lib, mb.MAP_EINVAL, mb.MAP_EUNSUPPORTED
    h, c = heads(mb, n=2, row=128), cache(mb)
    for bad, code in ((dict(pool=0), E), (dict(pool=F + 8), E), (dict(table=0), E), (dict(length=0), E), (dict(refs=0), E),
                      (dict(status=0), E), (dict(typ=2), E), (dict(layers=0), E), (dict(pages=0), E), (dict(hk=0), E),
                      (dict(page=0), E), (dict(dh=0), E), (dict(seqs=0), E), (dict(max_pages=0), E), (dict(dh=60), U),
                      (dict(dh=264), U), (dict(page=1025), U), (dict(seqs=262145), U), (dict(pages=(1 << 20) + 1), U),
                      (dict(max_pages=1 << 27), U)):
        b = cache(mb, **bad)
        assert lib.map_cache_free(b, F, 1, None) == code, bad
        assert lib.map_cache_extend(b, F, F, 1, 1, F, None) == code
        assert lib.map_cache_fork(b, F, F, 1, None, 0, None, None, None) == code
        assert lib.map_cache_attend(b, 0, h, F, 1, 1.0, h, F, None) == code
        assert lib.map_cache_status(b, None) == code
        assert lib.map_qk_rotate_append(rope.h, b, 0, 1, F, F, h, h, h, None, None, h, None) == code
        assert lib.map_cache_attend_workspace(b) == 0
    assert lib.map_cache_free(c, None, 1, None) == E
    assert lib.map_cache_free(c, F, -1, None) == E
    assert lib.map_cache_free(c, F, (1 << 20) + 1, None) == U
    assert lib.map_cache_free(c, None, 0, None) == mb.MAP_OK
    assert lib.map_cache_extend(c, None, F, 1, 1, F, None) == E
    assert lib.map_cache_extend(c, F, F, 1, 1, None, None) == E
    assert lib.map_cache_extend(c, F, F, 1, -1, F, None) == E
    assert lib.map_cache_extend(c, F, F, 4097, 1, F, None) == U
    assert lib.map_cache_extend(c, F, F, 1, (1 << 20) + 1, F, None) == U
    assert lib.map_cache_fork(c, None, F, 1, None, 0, None, None, None) == E
    assert lib.map_cache_fork(c, F, F, 1, F, 2, None, None, None) == E                # keep without its window
    assert lib.map_cache_fork(c, F, F, 1, F, 2, F, None, None) == E
    assert lib.map_cache_fork(c, F, F, 1, None, 2, F, F, None) == E
    assert lib.map_cache_fork(c, F, F, 1, F, -1, F, F, None) == E
    assert lib.map_cache_fork(c, F, F, 4097, F, 2, F, F, None) == U
    A = lib.map_qk_rotate_append
    assert A(rope.h, c, 2, 1, F, F, h, h, h, None, None, h, None) == E                # layer
    assert A(rope.h, c, -1, 1, F, F, h, h, h, None, None, h, None) == E
    assert A(rope.h, c, 0, 1, F, None, h, h, h, None, None, h, None) == E             # slots
    assert A(rope.h, c, 0, 1, None, F, h, h, h, None, None, h, None) == E             # positions
    assert A(rope.h, c, 0, 1, F, F, h, heads(mb, n=4), h, None, None, h, None) == E   # key heads
    assert A(rope.h, c, 0, 1, F, F, h, h, None, None, None, h, None) == E
    assert A(rope.h, c, 0, 1, F, F, h, h, h, None, None, None, None) == E             # q without an output
    assert A(rope.h, cache(mb, dh=128), 0, 1, F, F, h, h, h, None, None, h, None) == E
    T = lib.map_cache_attend
    assert T(c, 2, h, F, 1, 1.0, h, F, None) == E
    assert T(c, 0, heads(mb, n=3), F, 1, 1.0, heads(mb, n=3), F, None) == E           # 3 heads over 2
    assert T(c, 0, h, F, 1, math.nan, h, F, None) == E
    assert T(c, 0, h, F, 1, math.inf, h, F, None) == E
    assert T(c, 0, h, None, 1, 1.0, h, F, None) == E
    assert T(c, 0, h, F, 1, 1.0, h, None, None) == E
    assert T(c, 0, heads(mb, n=2, p=F + 2), F, 1, 1.0, h, F, None) == E
    assert T(c, 0, heads(mb, n=2, row=129), F, 1, 1.0, h, F, None) == E
    assert T(c, 0, h, F, 2, 1.0, heads(mb, n=2, row=64, head=64), F, None) == E       # overlapping outputs
    h72 = heads(mb, n=2, row=144, head=72)
    assert T(cache(mb, dh=72), 0, h72, F, 1, 1.0, h72, F, None) == U
    assert T(c, 0, h, F, 65536, 1.0, h, F, None) == U
    assert T(c, 0, h, None, 0, 1.0, h, None, None) == mb.MAP_OK


def test_cache_limits_of_a_page(mb):
    """heads, and the units (planes times heads) that a page is copied in, are counted in 32 bits."""
    free, E = mb.lib.map_cache_free, mb.MAP_EUNSUPPORTED
    assert free(cache(mb, hk=65535, layers=128), None, 0, None) == mb.MAP_OK
    assert free(cache(mb, hk=1, layers=1 << 23), None, 0, None) == mb.MAP_OK
    for bad in (dict(hk=65536), dict(hk=65535, layers=129), dict(hk=1, layers=(1 << 23) + 1), dict(hk=65535, layers=1 << 30)):
        assert free(cache(mb, **bad), None, 0, None) == E, bad


def test_calls_without_any_heads(mb, rope):
    with pytest.raises(ValueError):
        rope.rotate(None, None, None)
    with pytest.raises(ValueError):
        rope.grad(None, None, None)


def test_assemble_axes_refusals(mb):
    lib, E = mb.lib, mb.MAP_EINVAL
    lens = (ctypes.c_int32 * 1)(3)

    def call(ctx=F, lens=lens, grid=(2, 2, 2), step=None, B=1, N=8, k=2, off=0):
        g = (ctypes.c_int32 * 3)(*grid) if grid else None
        s = (ctypes.c_int32 * 1)(step) if step is not None else None
        return lib.map_assemble_axes(ctx, F, F, F, lens, g, s, B, N, k, off, F, F, None)

    for bad in (dict(ctx=None), dict(lens=None), dict(grid=None), dict(lens=(ctypes.c_int32 * 1)(-1)), dict(B=0), dict(N=0),
                dict(k=-1), dict(k=9), dict(grid=(0, 2, 2)), dict(grid=(3, 2, 2)), dict(grid=(1, 2, 2), k=5),
                dict(grid=(1 << 20, 1 << 20, 1 << 20)), dict(step=-1)):
        assert call(**bad) == E, bad
    assert call(step=0x7fffffff) == mb.MAP_EUNSUPPORTED
    assert call(off=0x7fffffff) == mb.MAP_EUNSUPPORTED


# ----------------------------------------------------------------------------- the models

def test_axis_positions_hand_example():
    # a 2 x 2 x 3 video, frames two positions apart: tokens 0, 5 and 10; two question tokens after max(3, 2, 3)
    got = H.axis_positions([[0, 5, 10]], [2], [(2, 2, 3)], [2], pos_offset=7)
    assert got.tolist() == [[7, 7, 9, 10, 11], [7, 8, 8, 10, 11], [7, 9, 8, 10, 11]]


def test_rotation_of_hand_values():
    x = np.array([[[1.0, 0.0, 3.0, 4.0, 9.0]]])
    y, _ = H.rotate(x, None, [[2], [0]], [math.pi / 4, 1.0], [0, 1], True, 0.0)          # first pair a quarter turn
    assert np.allclose(y, [[[0.0, 1.0, 3.0, 4.0, 9.0]]])
    y, _ = H.rotate(x, None, [[2], [0]], [math.pi / 4, 1.0], [0, 1], False, 0.0)         # pairs (0, 2) and (1, 3)
    assert np.allclose(y, [[[-3.0, 0.0, 1.0, 4.0, 9.0]]])
    y, z = H.rotate(np.array([[[3.0, 4.0]]]), np.array([2.0, 1.0]), [[0]], [1.0], [0], False, 0.0)
    assert np.allclose(y, np.array([6.0, 4.0]) / math.sqrt(12.5)) and np.allclose(y, z)


@pytest.mark.parametrize("adjacent,norm", [(False, True), (True, True), (False, False)])
def test_rotation_gradient_against_differences(adjacent, norm):
    rng = np.random.default_rng(5)
    x, dy, w = rng.normal(size=(3, 2, 10)), rng.normal(size=(3, 2, 10)), 1 + 0.3 * rng.normal(size=10)
    pos, f, ax = rng.integers(-50, 50, size=(2, 3)), [0.9, 0.31, 0.07, 0.011], [0, 1, 1, 0]
    w = w if norm else None

    def loss(x, w):
        return (H.rotate(x, w, pos, f, ax, adjacent, 1e-3)[0] * dy).sum()

    dx, dw = H.rotate_grad(dy, x, w, pos, f, ax, adjacent, 1e-3)
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-6
        assert abs((loss(x + e, w) - loss(x - e, w)) / 2e-6 - dx[i]) < 1e-7
    for c in range(10 if norm else 0):
        e = np.zeros(10)
        e[c] = 1e-6
        assert abs((loss(x, w + e) - loss(x, w - e)) / 2e-6 - dw[c]) < 1e-7


def test_pages_model_by_hand():
    m = H.Pages(6, 2, 4, 4)
    assert m.extend([2, -1, 0], [3, 7, 1], 6) == [0, 1, 2, 4, -1, -1]
    assert H.Pages(3, 2, 4, 4).extend([1, -1, 0], None, 4) == [0, -1, 2, -1] and m.extend([1, 3], None, 1) is None
    assert m.extend([2, 2], [1, 1], 2) is None and m.extend([1], [9], 9) is None and m.extend([1], [2], 1) is None
    assert m.fork([2, 2], [1, 3], [[0], [0]], [1, 0], [1, 3]) == [(6, 0), (7, 1), (8, 2), (10, 0)]
    m2 = H.Pages(6, 2, 4, 4)
    m2.extend([0], [5], 5)
    assert m2.fork([0], [1]) == [(6, 4)] and m2.table[1] == [0, 1, 3] and m2.refs == [2, 2, 1, 1, 0, 0]
    m2.free([0, 0, -1])
    assert m2.refs == [1, 1, 0, 1, 0, 0] and m2.extend([2], [3], 3) == [4, 5, 8]
    assert m2.fork([1], [1]) is None and m2.fork([9], [3]) is None and m2.fork([1], [2]) is None
