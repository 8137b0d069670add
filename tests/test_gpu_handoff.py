"""The language-model hand-off on the GPU against the 64-bit models of oracle/handoff_oracle.py.

Tolerances.  u = eps / 2 of the output's type is its one rounding.  Rotation: z = x r w carries the error of r (rsqrtf
2 ulp, a sum of dh squares in at most 16 + 8 steps, halved by the root, the division and eps: 2 + 12 + 2) and of two
products; cos and sin carry their argument's rounding, pi 2^-24, and 2 ulp; the turn adds 3 roundings: under 32 * 2^-24
of |z_a| + |z_b|.  fp16 results below 2^-14 are rounded to multiples of 2^-24.
"""
import os
import subprocess
import sys
import threading
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import handoff_oracle as H
from oracle import map_oracle as O

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
E24 = 2.0 ** -24


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_06411_gb300 import binding
    return binding


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def half_step(typ):
    return torch.finfo(typ).eps / 2


def tiny(typ):
    return 2.0 ** -25 if typ == torch.float16 else 1e-37


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, typ):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(typ)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ----------------------------------------------------------------------------- layouts

def place(x, layout):
    """A tensor of x's values laid out as `layout` says, and the storage it is a view of."""
    rows, heads, dh = x.shape
    if layout == "dense":
        base = x.clone()
        return base, base
    if layout == "packed":                       # between other columns of a projection's row
        base = torch.full((rows, (heads + 3) * dh), 7.0, dtype=x.dtype, device=x.device)
        view = base[:, 2 * dh: (2 + heads) * dh].unflatten(1, (heads, dh))
    elif layout == "heads_first":
        base = torch.full((heads, rows, dh), 7.0, dtype=x.dtype, device=x.device)
        view = base.transpose(0, 1)
    else:                                        # "odd": odd offset and strides
        base = torch.full((rows * (heads * (dh + 3) + 5) + 1,), 7.0, dtype=x.dtype, device=x.device)
        view = base[1:].as_strided((rows, heads, dh), (heads * (dh + 3) + 5, dh + 3, 1), 1)
    view.copy_(x)
    return view, base


ROTATIONS = [
    # type, rows, hq, hk, dh, rot, axes, adjacent, norm, layout, far
    ("bf16", 1, 28, 4, 128, 128, 3, False, True, "packed", 5000),
    ("bf16", 37, 8, 2, 128, 128, 3, True, True, "dense", 5000),
    ("f16", 130, 4, 4, 64, 32, 1, False, True, "heads_first", 5000),
    ("f32", 65, 5, 1, 80, 80, 2, False, True, "packed", 5000),
    ("f32", 19, 16, 16, 72, 72, 2, True, False, "dense", 60),
    ("f32", 19, 16, 3, 72, 72, 2, False, True, "dense", 60),
    ("bf16", 33, 3, 3, 96, 96, 4, False, False, "odd", 5000),
    ("bf16", 9, 1, 1, 256, 256, 3, False, True, "dense", 2 ** 31),
    ("f32", 9, 2, 1, 256, 128, 3, True, True, "heads_first", 2 ** 31),
    ("f16", 21, 2, 2, 37, 36, 2, False, True, "dense", 5000),
    ("bf16", 21, 2, 2, 37, 2, 2, True, True, "odd", 5000),
    ("f32", 7, 3, 2, 1, 0, 1, False, True, "dense", 5000),
    ("f16", 7, 3, 2, 20, 20, 3, False, True, "odd", 5000),
    ("bf16", 7, 3, 2, 20, 12, 3, True, True, "packed", 5000),
    ("bf16", 7, 3, 2, 48, 24, 3, False, False, "packed", 5000),
    ("f16", 700, 7, 1, 192, 64, 2, False, True, "packed", 100000),
    ("bf16", 2500, 32, 32, 128, 128, 3, False, True, "packed", 8192),
    ("f32", 1027, 4, 4, 128, 96, 2, False, False, "packed", 8192),
    ("f32", 3, 1, 2, 254, 254, 1, False, True, "dense", 8192),
    ("bf16", 1601, 56, 8, 36, 36, 3, False, True, "dense", 8192),
    ("f16", 801, 9, 2, 72, 36, 2, False, True, "packed", 8192),
    ("bf16", 300, 13, 4, 256, 256, 2, False, True, "odd", 8192),
    ("bf16", 301, 70, 5, 9, 8, 1, True, True, "odd", 8192),
]
IDS = ["-".join(str(v) for v in c) for c in ROTATIONS]


def rotation(mb, case, seed=1):
    typ, rows, hq, hk, dh, rot, axes, adjacent, norm, layout, far = case
    typ, g = TYPES[typ], gen(seed)
    q, k = randn(g, rows, hq, dh, typ=typ) * 2, randn(g, rows, hk, dh, typ=typ) * 2
    wq, wk = ((1 + 0.3 * torch.randn(dh, generator=g, device=DEV)).to(typ) for _ in range(2)) if norm else (None, None)
    pos = torch.randint(-far, far, (axes, rows), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    half = rot // 2
    inv = [10000.0 ** (-2.0 * i / max(rot, 1)) for i in range(half)]
    ax = [i % axes if adjacent else i * axes // max(half, 1) for i in range(half)]
    plan = mb.Rope(dh, inv, axis=ax, n_axes=axes, adjacent=adjacent, eps=1e-6)
    return typ, q, k, wq, wk, pos, inv, ax, plan


def check_rotated(got, x, w, pos, inv, ax, adjacent, typ):
    y, z = H.rotate(f64(x), f64(w), pos.cpu().numpy(), inv, ax, adjacent, 1e-6)
    size = np.abs(z)
    a, b = H.pairs_of(2 * len(inv), adjacent)
    both = size[..., a] + size[..., b]
    size[..., a], size[..., b] = both, both
    off = np.abs(f64(got) - y)
    tol = half_step(typ) * np.abs(y) * 1.001 + 32 * E24 * size + tiny(typ)
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("case", ROTATIONS, ids=IDS)
def test_rotate_matches_the_formula(mb, case):
    typ, q, k, wq, wk, pos, inv, ax, plan = rotation(mb, case)
    layout, adjacent = case[9], case[7]
    (qv, _), (kv, _) = place(q, layout), place(k, layout)
    (qo, qbase), (ko, kbase) = place(torch.full_like(q, 7.0), layout), place(torch.full_like(k, 7.0), layout)
    plan.rotate(qv, kv, pos, wq, wk, qo, ko)
    check_rotated(qo, q, wq, pos, inv, ax, adjacent, typ)
    check_rotated(ko, k, wk, pos, inv, ax, adjacent, typ)
    got_q, got_k = qo.clone(), ko.clone()
    qo.fill_(7.0), ko.fill_(7.0)                     # nothing but the heads was written
    assert bool((qbase == 7.0).all()) and bool((kbase == 7.0).all())
    assert torch.equal(qv, q) and torch.equal(kv, k)
    plan.rotate(qv, kv, pos, wq, wk, qv, kv)         # in place: the same
    assert torch.equal(qv, got_q) and torch.equal(kv, got_k)
    only_q, none = plan.rotate(q, None, pos, wq)     # one side alone, dense
    assert none is None
    check_rotated(only_q, q, wq, pos, inv, ax, adjacent, typ)
    none, only_k = plan.rotate(None, k, pos, None, wk)
    assert none is None
    check_rotated(only_k, k, wk, pos, inv, ax, adjacent, typ)


def test_rotate_edges(mb):
    inv = [0.5, 0.25]
    plan = mb.Rope(8, inv, axis=[0, 1], n_axes=2)
    pos = ints([[2 ** 31 - 1, -2 ** 31, 0], [5, 6, 7]])
    x = torch.randn(3, 2, 8, device=DEV)
    x[1, 0, 3] = float("nan")
    x[2, 1] = float("inf")
    y, _ = plan.rotate(x, None, pos, torch.ones(8, device=DEV))
    assert bool(torch.isnan(y[1, 0]).all()) and bool(torch.isnan(y[2, 1]).all())      # a bad head spoils itself alone
    keep = torch.ones(3, 2, dtype=torch.bool)
    keep[1, 0] = keep[2, 1] = False
    assert bool(torch.isfinite(y[keep.to(DEV)]).all())
    y, z = H.rotate(f64(x[:1]), None, pos.cpu().numpy()[:, :1], inv, [0, 1], False, 0.0)
    got, _ = plan.rotate(x[:1], None, pos[:, :1].contiguous())
    assert np.abs(f64(got) - y).max() < 1e-5
    for adjacent in (False, True):                                   # columns past rot do not touch each other
        for extra in (0, 1):                                         # (vectors, and any alignment)
            wide = mb.Rope(64, [0.5] * 16, adjacent=adjacent)
            x = torch.ones(2 * 64 + extra, device=DEV)[extra:].view(2, 1, 64)
            x[0, 0, 40] = float("inf")
            y, _ = wide.rotate(x, None, ints([[3, 4]]))
            assert int(torch.isfinite(y).sum()) == 127 and bool(torch.isinf(y[0, 0, 40]))
            y = wide.grad(x, None, ints([[3, 4]]))[0]
            assert int(torch.isfinite(y).sum()) == 127 and bool(torch.isinf(y[0, 0, 40]))
    x = torch.randn(3, 2, 8, device=DEV)
    back = mb.Rope(64, [-0.5, 0.0, -1e-30, 1e-30], axis=[0, 0, 0, 0])     # turned the other way, not, and hardly
    x = torch.randn(2, 1, 64, device=DEV)
    y, z = H.rotate(f64(x), None, [[3, 2 ** 31 - 1]], [-0.5, 0.0, -1e-30, 1e-30], [0] * 4, False, 0.0)
    got, _ = back.rotate(x, None, ints([[3, 2 ** 31 - 1]]))
    assert np.abs(f64(got) - y).max() < 1e-5
    x = torch.randn(3, 2, 8, device=DEV)
    for rows in (0,):
        q, k = plan.rotate(x[:rows], x[:rows], pos[:, :rows].contiguous())
        assert q.shape == (0, 2, 8) and k.shape == (0, 2, 8)
    # heads broadcast over rows are a valid input
    one = x[:1].expand(3, 2, 8)
    got, _ = plan.rotate(one, None, pos)
    want, _ = plan.rotate(one.contiguous(), None, pos)
    assert torch.equal(got, want)
    with pytest.raises(mb.MapError):
        plan.rotate(x, None, pos, q_out=torch.empty(1, 2, 8, device=DEV).expand(3, 2, 8))
    with pytest.raises(ValueError):
        plan.rotate(x, None, pos[:1])
    with pytest.raises(ValueError):
        plan.rotate(x, x.half(), pos)
    with pytest.raises(ValueError):
        plan.rotate(x.transpose(1, 2), None, pos)
    with pytest.raises(ValueError):
        plan.rotate(x.double(), None, pos)


def test_rotation_angles_at_far_positions(mb):
    """Angles from rational arithmetic with 50 digits of 2 pi: cut to 32 bits they are off by 2^-32 turns, and by |pos| 2^-65 of
    the stored fraction's rounding, together under 2^-29 radians; the rest as above."""
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    inv = [1000.0, 37.5, 1.0, 123456.789, 0.1, 3e9, -777.25, 1e-3, 2.0 ** 40 + 0.125, 6.283185307179586, 0.5, -2.5]
    at = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 1999999999, -1234567891, 7]
    plan = mb.Rope(32, inv)
    x = randn(gen(1), len(at), 2, 32, typ=torch.float32)
    for v in (x, place(x, "odd")[0]):
        got = f64(plan.rotate(v, None, ints([at]))[0])
        for r, p in enumerate(at):
            for i, f in enumerate(inv):
                t = p * Fraction(f) / two_pi
                t = float((t - int(t)) * two_pi)
                a, b = f64(x[r, :, i]), f64(x[r, :, len(inv) + i])
                size = (32 * E24 + 2.0 ** -29) * (np.abs(a) + np.abs(b))
                assert (np.abs(got[r, :, i] - (a * np.cos(t) - b * np.sin(t))) <= size).all(), (p, f)
                assert (np.abs(got[r, :, len(inv) + i] - (b * np.cos(t) + a * np.sin(t))) <= size).all(), (p, f)


def check_grad(dx, dw, dy, x, w, pos, inv, ax, adjacent, typ):
    """dx: r (g w - n mean(g w n)); errors as above, and of the mean: dh products in 24 steps and the roundings of both
    factors, 40 steps.  dw: a term's 24 steps (g 20 and n 3), and the additions of its sum, each at most 2^-24 of the sum
    of magnitudes: rows * heads / (blocks * heads in flight) in a thread, under 64, 32 heads of a block and 608 blocks."""
    x64, w64, p = f64(x), f64(w), pos.cpu().numpy()
    want, wdw = H.rotate_grad(f64(dy), x64, w64, p, inv, ax, adjacent, 1e-6)
    g = np.abs(H.rotate(f64(dy), None, p, -np.asarray(inv), ax, adjacent, 0.0)[0])
    size = np.abs(f64(dy))
    a, b = H.pairs_of(2 * len(inv), adjacent)
    both = size[..., a] + size[..., b]
    size[..., a], size[..., b] = both, both                      # bounds g
    if w is not None:
        r = 1 / np.sqrt((x64 ** 2).mean(-1, keepdims=True) + 1e-6)
        n = np.abs(x64 * r)
        gsize = size
        size = r * (gsize * np.abs(w64) + n * (gsize * np.abs(w64) * n).mean(-1, keepdims=True))
    tol = half_step(typ) * np.abs(want) * 1.001 + 64 * E24 * size + tiny(typ)
    off = np.abs(f64(dx) - want)
    assert (off <= tol).all(), float((off / tol).max())
    if w is not None:
        tol = (24 + 64 + 32 + 608) * E24 * (gsize * n).sum((0, 1)) + 1e-37
        off = np.abs(f64(dw) - wdw)
        assert (off <= tol).all(), float((off / tol).max())
    else:
        assert dw is None


@pytest.mark.parametrize("case", ROTATIONS, ids=IDS)
def test_rotate_grad_matches_the_formula(mb, case):
    typ, q, k, wq, wk, pos, inv, ax, plan = rotation(mb, case)
    layout, adjacent = case[9], case[7]
    g = gen(9)
    dq, dk = randn(g, *q.shape, typ=typ), randn(g, *k.shape, typ=typ)
    (qv, _), (kv, _), (dqv, _), (dkv, _) = (place(t, layout) for t in (q, k, dq, dk))
    (qo, qbase), (ko, kbase) = place(torch.full_like(q, 7.0), layout), place(torch.full_like(k, 7.0), layout)
    _, _, dwq, dwk = plan.grad(dqv, dkv, pos, qv, kv, wq, wk, dq=qo, dk=ko)
    check_grad(qo, dwq, dq, q, wq, pos, inv, ax, adjacent, typ)
    check_grad(ko, dwk, dk, k, wk, pos, inv, ax, adjacent, typ)
    a, b = qo.clone(), ko.clone()
    again = plan.grad(dqv, dkv, pos, qv, kv, wq, wk, dq=qo, dk=ko)   # the same again, sums too (fixed order)
    assert torch.equal(a, qo) and torch.equal(b, ko)
    assert wq is None or torch.equal(dwq, again[2]) and torch.equal(dwk, again[3])
    dense = plan.grad(dq, dk, pos, q, k, wq, wk)
    check_grad(dense[0], dense[2], dq, q, wq, pos, inv, ax, adjacent, typ)
    check_grad(dense[1], dense[3], dk, k, wk, pos, inv, ax, adjacent, typ)
    qo.fill_(7.0), ko.fill_(7.0)
    assert bool((qbase == 7.0).all()) and bool((kbase == 7.0).all())
    plan.grad(dqv, dkv, pos, qv, kv, wq, wk, dq=dqv, dk=dkv)         # in place
    assert torch.equal(dqv, a) and torch.equal(dkv, b)


@pytest.mark.parametrize("typ,dh,layout,top", [("bf16", 128, "dense", 1.4e18), ("f32", 128, "dense", 1.4e18),
                                               ("bf16", 64, "dense", 2e18), ("f32", 256, "dense", 1e18), ("bf16", 8, "dense", 6e18),
                                               ("f32", 128, "odd", 1.4e18), ("bf16", 36, "odd", 2.9e18), ("bf16", 6, "dense", 6e18)])
def test_norms_of_heads_whose_squares_almost_overflow(mb, typ, dh, layout, top):
    """The sum of a head's squares is below 2^128, 32 / lanes times it is not."""
    typ, g, rows, heads = TYPES[typ], gen(3), 33, 3
    inv = [0.9 ** i for i in range(dh // 2)]
    x = (randn(g, rows, heads, dh, typ=torch.float32).sign() * top * (1 - 0.2 * torch.rand(rows, heads, dh, generator=g, device=DEV))).to(typ)
    assert float(x.double().square().sum(-1).max()) < 3.3e38
    dy = randn(g, rows, heads, dh, typ=typ)
    w = (1 + 0.3 * torch.randn(dh, generator=g, device=DEV)).to(typ)
    pos = torch.randint(0, 5000, (1, rows), generator=g, device=DEV, dtype=torch.int32)
    plan = mb.Rope(dh, inv)
    (xv, _), (dyv, _) = place(x, layout), place(dy, layout)
    y, _ = plan.rotate(xv, None, pos, w)
    check_rotated(y, x, w, pos, inv, [0] * len(inv), False, typ)
    dx, _, dw, _ = plan.grad(dyv, None, pos, xv, None, w)
    check_grad(dx, dw, dy, x, w, pos, inv, [0] * len(inv), False, typ)


def test_rotate_grad_against_differences(mb):
    """<grad, d> = (loss(x + h d) - loss(x - h d)) / 2h in fp32: the difference is off by h^2 / 6 of the third derivative
    (of order 10 for heads of unit norm: 2e-4 at h = 1e-2 times the sum's size) and by fp32 roundings over h (a sum of
    1e3 terms of size 1: 1e3 * 2^-24 * 32 / 1e-2 = 0.2 of a gradient of size 30)."""
    rows, heads, dh = 5, 3, 64
    inv = [10000.0 ** (-2.0 * i / dh) for i in range(dh // 2)]
    plan = mb.Rope(dh, inv, axis=[i % 3 for i in range(dh // 2)])
    g = gen(3)
    x, dy, d, w = (randn(g, rows, heads, dh, typ=torch.float32) for _ in range(4))
    w = 1 + 0.2 * w[0, 0]
    pos = torch.randint(0, 500, (3, rows), generator=g, device=DEV, dtype=torch.int32)
    dx, _, dw, _ = plan.grad(dy, None, pos, x, None, w)
    h = 1e-2

    def loss(x, w):
        return float((plan.rotate(x, None, pos, w)[0].double() * dy.double()).sum())

    num = (loss(x + h * d, w) - loss(x - h * d, w)) / (2 * h)
    assert abs(num - float((dx.double() * d.double()).sum())) < 0.3
    e = d[0, 0]
    num = (loss(x, w + h * e) - loss(x, w - h * e)) / (2 * h)
    assert abs(num - float((dw.double() * e.double()).sum())) < 0.3


def test_rotate_grad_of_no_rows_and_one_side(mb):
    plan = mb.Rope(64, [1.0] * 32)
    z = torch.zeros(0, 2, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    pos = torch.zeros(1, 0, dtype=torch.int32, device=DEV)
    dq, dk, dwq, dwk = plan.grad(z, None, pos, z, None, w, dwq=torch.full((64,), 3.0, device=DEV))
    assert dk is None and dwk is None and dq.shape == z.shape and bool((dwq == 0).all())


@pytest.mark.parametrize("typ,dh,adjacent", [("bf16", 80, False), ("bf16", 96, False), ("f16", 192, False), ("f16", 48, False),
                                             ("f32", 80, False), ("f32", 72, False), ("f16", 20, False), ("bf16", 80, True),
                                             ("f32", 12, True)])
def test_rotate_grad_after_sums_of_nan(mb, typ, dh, adjacent):
    """Heads whose vectors are no power of two leave lanes without columns.  What an earlier kernel left in shared memory
    must not reach their heads' sums: a gradient of NaN, 256 columns wide, leaves sums of NaN there."""
    typ, g, rows, heads = TYPES[typ], gen(3), 1200, 4
    inv = [0.9 ** i for i in range(dh // 2)]
    x, dy = (randn(g, rows, heads, dh, typ=typ) for _ in range(2))
    w = (1 + 0.3 * torch.randn(dh, generator=g, device=DEV)).to(typ)
    pos = torch.randint(0, 5000, (1, rows), generator=g, device=DEV, dtype=torch.int32)
    wide = torch.full((rows, heads, 256), float("nan"), dtype=typ, device=DEV)
    bad, plan = (mb.Rope(d, f, adjacent=adjacent) for d, f in ((256, [1.0] * 128), (dh, inv)))
    assert bool(torch.isnan(bad.grad(wide, None, pos, wide, None, wide[0, 0])[2]).all())
    dx, _, dw, _ = plan.grad(dy, None, pos, x, None, w)
    check_grad(dx, dw, dy, x, w, pos, inv, [0] * len(inv), adjacent, typ)


def test_rotate_grad_of_a_side_without_heads(mb):
    plan, pos = mb.Rope(64, [1.0] * 32), ints([[1, 2, 3, 4, 5]])
    none, x, dy = torch.zeros(5, 0, 64, device=DEV), *(randn(gen(s), 5, 2, 64, typ=torch.float32) for s in (1, 2))
    w = torch.ones(64, device=DEV)
    alone = plan.grad(None, dy, pos, None, x, None, w)
    for sides in (0, 1):
        d = torch.full((64,), 3.0, device=DEV)
        got = plan.grad(none, dy, pos, none, x, w, w, dwq=d) if sides == 0 else plan.grad(dy, none, pos, x, none, w, w, dwk=d)
        assert bool((d == 0).all())
        assert torch.equal(got[2 + (1 - sides)], alone[3])


# ----------------------------------------------------------------------------- positions

@pytest.mark.parametrize("grids,lens,k,step,off,N", [
    ([(1, 24, 24)], [32], 32, None, 0, 576),
    ([(1, 24, 24), (4, 6, 5), (3, 1, 40), (1, 1, 33)], [5, 0, 77, 1], 33, [1, 3, 0, 9], 35, 600),
    ([(2, 3, 4)] * 3, [2, 0, 1], 0, [2, 2, 2], -3, 24),
    ([(1, 2, 3)], [0], 6, None, 0, 6),
    ([(2, 2, 2)] * 700, [i % 3 for i in range(700)], 3, list(range(700)), 1, 8),
])
def test_assemble_axes(mb, grids, lens, k, step, off, N):
    D, B = 512, len(grids)
    ctx = handoff_context(mb, D)
    rng = np.random.default_rng(3)
    vis = rng.integers(0, 2 ** 16, size=(B, N, D), dtype=np.uint16)
    text = rng.integers(0, 2 ** 16, size=(max(1, sum(lens)), D), dtype=np.uint16)
    keep = np.stack([np.sort(rng.choice(t * h * w, k, replace=False)) for t, h, w in grids]).astype(np.int32)
    seq, pos = ctx.assemble_axes(torch.from_numpy(vis.view(np.int16)).to(DEV), torch.from_numpy(keep).to(DEV),
                                 torch.from_numpy(text.view(np.int16)).to(DEV), lens, grids, step, off)
    ctx.check()
    ref, _ = O.assemble(vis, keep, text[: sum(lens)], lens)
    np.testing.assert_array_equal(seq.cpu().numpy().view(np.uint16), ref)
    np.testing.assert_array_equal(pos.cpu().numpy(), H.axis_positions(keep, lens, grids, step, off))


def test_assemble_axes_reports_a_bad_index(mb):
    ctx = handoff_context(mb, 512)
    vis, text = torch.zeros((2, 9, 512), dtype=torch.int16, device=DEV), torch.ones((2, 512), dtype=torch.int16, device=DEV)
    seq = torch.full((6, 512), 5, dtype=torch.int16, device=DEV)
    _, pos = ctx.assemble_axes(vis, ints([[0, 8], [6, -1]]), text, [1, 1], [(2, 2, 2), (1, 3, 3)], seq=seq)
    assert ctx.status() == mb.MAP_EINTERNAL and ctx.status() == mb.MAP_OK
    assert pos.cpu().tolist() == [[0, -1, 2, 0, -1, 3], [0, -1, 2, 2, -1, 3], [0, -1, 2, 0, -1, 3]]
    assert seq[:, 0].cpu().tolist() == [0, 5, 1, 0, 5, 1]
    with pytest.raises(ValueError):
        ctx.assemble_axes(vis, ints([[0, 8], [6, -1]]), text, [1, 1], [(2, 2, 2)])


_CONTEXTS = {}


def handoff_context(mb, D):
    if D not in _CONTEXTS:
        shapes = {"wT1": (256, D), "bT1": (256,), "wT2": (256, 256), "bT2": (256,), "wQ": (64, 256)}
        shapes.update({n.replace("T", "V").replace("Q", "K"): s for n, s in shapes.items()})
        _CONTEXTS[D] = mb.Context({n: torch.zeros(s, dtype=torch.int16, device=DEV) for n, s in shapes.items()}, D, 256, 64)
    return _CONTEXTS[D]


# ----------------------------------------------------------------------------- pages

def rows_of(pool, slots):
    """[layers, 2, rows, heads, dh] at the given slots."""
    page = pool.shape[4]
    s = torch.tensor(slots, dtype=torch.int64, device=pool.device)
    return pool[:, :, s // page, :, s % page].permute(1, 2, 0, 3, 4) if len(slots) else pool[:, :, :0, 0, 0]


def same_state(cache, model):
    assert cache.length.cpu().tolist() == model.length
    assert cache.refs.cpu().tolist() == model.refs
    table = cache.table.cpu().tolist()
    for s, pages in enumerate(model.table):
        assert table[s][: len(pages)] == pages, s


@pytest.mark.parametrize("page,dh,hk,layers,seed", [(16, 128, 2, 2, 0), (1, 8, 1, 1, 1), (5, 40, 3, 2, 2), (64, 64, 8, 1, 3),
                                                    (1024, 16, 1, 1, 4), (7, 256, 1, 3, 5)])
def test_page_calls_follow_the_model(mb, page, dh, hk, layers, seed):
    """A long run of extensions, appended rows, forks, pruned forks and frees, good and refused ones."""
    import random
    r = random.Random(seed)
    pages, seqs, max_pages = r.randint(20, 45), 9, 8
    cache = mb.Cache.empty(layers, pages, hk, page, dh, seqs, max_pages, torch.float16)
    cache.pool.normal_(generator=gen(seed))
    model = H.Pages(pages, page, seqs, max_pages)
    plan = mb.Rope(dh, [0.3, 0.1], n_axes=1)
    refused = copied = 0
    for step in range(120):
        op = r.choice(["extend", "extend", "fork", "prune", "free"])
        before = cache.pool.clone()
        if op == "extend":
            n = r.randint(0, 4)
            who = [r.choice([-1] + list(range(seqs))) if r.random() < 0.97 else r.choice([seqs, -2]) for _ in range(n)]
            counts = [r.choice([0, 1, 1, page, r.randint(0, 2 * page + 1)]) if r.random() < 0.97 else -1 for _ in range(n)]
            rows = max(0, sum(c for c, w in zip(counts, who) if w != -1)) + r.choice([0, 0, 3])
            rows = max(0, rows - (1 if r.random() < 0.05 else 0))
            if r.random() < 0.3:
                counts, rows = None, n + r.choice([0, 0, 2, -1 if n else 0])
            want = model.extend(who, counts, rows)
            got = cache.extend(ints(who), None if counts is None else ints(counts), rows=rows)
            assert got.cpu().tolist() == (want if want is not None else [-1] * rows)
            named = [w for w in who if w != -1]
            ok = want is not None
            if ok and rows and r.random() < 0.5:
                layer = r.randrange(layers)
                k, v, q = (randn(gen(step), rows, h, dh, typ=torch.float16) for h in (hk, hk, 2))
                pos = torch.arange(rows, dtype=torch.int32, device=DEV)[None]
                qo = torch.full_like(q, 3.0)
                plan.append(q, k, v, pos, cache, layer, got, q_out=qo)
                rq, rk = plan.rotate(q, k, pos)
                real = [i for i, s in enumerate(want) if s >= 0]
                pad = [i for i, s in enumerate(want) if s < 0]
                assert torch.equal(qo[real], rq[real]) and bool((qo[pad] == 3.0).all())
                at = torch.tensor([want[i] for i in real], dtype=torch.int64, device=DEV)
                before[layer, 0][at // page, :, at % page] = rk[real]
                before[layer, 1][at // page, :, at % page] = v[real]
        elif op in ("fork", "prune"):
            n = r.randint(0, 3)
            par = [r.randrange(seqs) if r.random() < 0.98 else seqs + 3 for _ in range(n)]
            empty = [s for s in range(seqs) if model.length[s] == 0]
            chi = [r.choice(empty) if empty and r.random() < 0.97 else r.randrange(seqs) for _ in range(n)]
            keep = base = span = None
            k = r.choice([0, 1, 2, page + 3])
            if op == "prune":
                base, span = [], []
                for p in par:
                    have = model.length[p] if p < seqs else 4
                    b = r.randint(0, have)
                    base.append(b if r.random() < 0.98 else -1)
                    span.append(r.randint(0, have - b) + (1 if r.random() < 0.02 else 0))
                keep = [[r.randint(0, max(0, s - 1)) if r.random() < 0.97 else s + 2 for _ in range(k)] for s in span]
            dev = [None if keep is None else ints(keep).reshape(n, k), *(None if x is None else ints(x) for x in (base, span))]
            want = model.fork(par, chi, keep, base, span)
            cache.fork(ints(par), ints(chi), *dev)
            ok = want is not None
            bad_index = ok and any(s < 0 for _, s in want)
            if ok:
                copied += len(want)
                for to, at in want:
                    src = 0.0 if at < 0 else before[:, :, at // page, :, at % page].clone()
                    before[:, :, to // page, :, to % page] = src
            if bad_index:
                assert cache.status() == mb.MAP_EINTERNAL
        else:
            who = [r.choice([-1] + list(range(seqs))) for _ in range(r.randint(0, 3))]
            model.free(who)
            cache.free(ints(who))
            ok = True
        if not ok:
            refused += 1
            assert cache.status() in (mb.MAP_ENOMEM, mb.MAP_EINTERNAL)
        assert cache.status() == mb.MAP_OK
        same_state(cache, model)
        assert torch.equal(cache.pool, before), (step, op)
    assert refused > 5 and copied > 5


def test_many_entries_and_a_large_pool(mb):
    """4096 sequences extended in one call, over pages whose free ones lie behind used ones; freed in one call."""
    n, page = 4096, 4
    cache = mb.Cache.empty(1, 40000, 1, page, 8, n + 2, 4)
    model = H.Pages(40000, page, n + 2, 4)
    first = [n, n + 1]
    assert cache.extend(ints(first), ints([16, 9]), rows=25).cpu().tolist() == model.extend(first, [16, 9], 25)
    counts = [(i * 7) % 14 for i in range(n)]
    got = cache.extend(ints(list(range(n))), ints(counts), rows=sum(counts) + 5).cpu().tolist()
    assert got == model.extend(list(range(n)), counts, sum(counts) + 5)
    same_state(cache, model)
    cache.free(ints(list(range(0, n, 2)) * 2 + [-1]))
    model.free(range(0, n, 2))
    got = cache.extend(ints(list(range(0, n, 2)))).cpu().tolist()
    assert got == model.extend(list(range(0, n, 2)), [1] * (n // 2), n // 2)
    same_state(cache, model)
    cache.check()


def test_bad_tables_and_lengths_are_reported_and_not_followed(mb):
    """Entries outside the pool and lengths outside a table row, in the caller's own arrays."""
    def fresh():
        c = mb.Cache.empty(1, 12, 2, 4, 64, 5, 3)
        c.pool.fill_(1.0)
        c.extend(ints([0, 1]), ints([10, 5]), rows=15)
        c.check()
        return c

    q = torch.ones(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    for page in (12, -1, 2 ** 31 - 1, -2 ** 31):
        c = fresh()
        c.table[0, 1] = page
        out = c.attend(q, ints([0, 1]), 0)
        assert c.status() == mb.MAP_EINTERNAL and bool((out == 1).all())
        c.fork(ints([0]), ints([2]), ints([[0]]), ints([0]), ints([1]))             # a copied row of the page
        assert c.status() == mb.MAP_EINTERNAL
        c.free(ints([2]))
        c.check()
        c.fork(ints([0]), ints([3]))                                                # the page shared
        assert c.status() == mb.MAP_EINTERNAL
        c.free(ints([0, 3]))
        assert c.status() == mb.MAP_EINTERNAL
        c = fresh()
        c.table[1, 1] = page                                                        # the part page that grows
        assert c.extend(ints([1])).cpu().tolist() == [-1]
        assert c.status() == mb.MAP_EINTERNAL
    for length in (-1, 13, 2 ** 31 - 1, -2 ** 31):
        c = fresh()
        c.length[0] = length
        before = c.refs.clone()
        assert c.extend(ints([0])).cpu().tolist() == [-1] and c.status() == mb.MAP_EINTERNAL
        c.fork(ints([0]), ints([2]))
        assert c.status() == mb.MAP_EINTERNAL and int(c.length[2]) == 0
        out = c.attend(q, ints([0, 1]), 0)
        assert c.status() == mb.MAP_EINTERNAL and bool((out[0] == 0).all()) and bool((out[1] == 1).all())
        assert torch.equal(c.refs, before)
        c.free(ints([0]))
        assert c.status() == mb.MAP_EINTERNAL and torch.equal(c.refs, before)


def test_free_leaves_a_bad_length_as_it_is(mb):
    for length in (-1, 13, 2 ** 31 - 1, -2 ** 31):
        c = mb.Cache.empty(1, 12, 2, 4, 64, 5, 3)
        c.extend(ints([0, 1]), ints([10, 5]), rows=15)
        c.length[0] = length
        c.free(ints([0, 1, 0, 1]))
        assert c.status() == mb.MAP_EINTERNAL
        assert c.length.cpu().tolist() == [length, 0, 0, 0, 0] and int(c.refs.sum()) == 3


def test_free_takes_the_good_entries_of_a_call(mb):
    """Free is the one page call that goes entry by entry: a bad sequence is reported, the others are freed."""
    c = mb.Cache.empty(1, 12, 2, 4, 64, 5, 3)
    c.extend(ints([0, 1, 4]), ints([10, 5, 1]), rows=16)
    c.free(ints([5, 0, -1, -7, 0, 4, 2]))
    assert c.status() == mb.MAP_EINTERNAL
    assert c.length.cpu().tolist() == [0, 5, 0, 0, 0] and c.refs.cpu().tolist() == [0, 0, 0, 1, 1] + [0] * 7


def test_forks_whose_pages_add_up_past_32_bits(mb):
    """A length that a very wide table row holds: 16 children of 2^27 pages each, of a pool of 64, are refused."""
    c = mb.Cache(torch.ones(1, 2, 64, 1, 1, 8, dtype=torch.float16, device=DEV),
                 torch.zeros(17, 1 << 27, dtype=torch.int32, device=DEV), ints([1 << 27] + [0] * 16), ints([0] * 64))
    children = ints(list(range(1, 17)))
    for n, code in ((16, mb.MAP_ENOMEM), (1, mb.MAP_ENOMEM)):
        c.fork(ints([0] * n), children[:n], torch.zeros(n, 0, dtype=torch.int32, device=DEV), ints([0] * n), ints([0] * n))
        assert c.status() == code
        assert int(c.length[1:].abs().sum()) == 0 and int(c.refs.abs().sum()) == 0 and int(c.table[1].abs().sum()) == 0


def test_lengths_just_below_32_bits(mb):
    """Lengths that a row of the table holds, where a page or a tile more passes 2^31: rows added, forked, freed, attended.
    (Every page of the long rows is page 0; its count says so.)"""
    long, cols = 2147482900, 2147483                                 # 2147483 pages of 1000
    pool = randn(gen(3), 1, 2, 4, 1, 1000, 8, typ=torch.float16)
    before = pool.clone()
    c = mb.Cache(pool, torch.zeros(3, cols, dtype=torch.int32, device=DEV), ints([long, 0, 0]), ints([cols, 0, 0, 0]))
    assert c.extend(ints([0])).cpu().tolist() == [900]
    assert c.length.cpu().tolist() == [long + 1, 0, 0] and c.refs.cpu().tolist() == [cols, 0, 0, 0]
    c.fork(ints([0]), ints([2]))
    c.check()
    assert c.length.cpu().tolist() == [long + 1, 0, long + 1] and c.refs.cpu().tolist() == [2 * cols - 1, 1, 0, 0]
    assert int(c.table[2, :-1].abs().max()) == 0 and int(c.table[2, -1]) == 1
    before[:, :, 1, :, :901] = before[:, :, 0, :, :901]
    assert torch.equal(pool, before)
    c.free(ints([2, 0]))
    c.check()
    assert c.length.cpu().tolist() == [0, 0, 0] and c.refs.cpu().tolist() == [0, 0, 0, 0]
    cols = 2 ** 27 - 1
    pool = torch.zeros(1, 2, 2, 1, 16, 64, dtype=torch.float16, device=DEV)
    pool[:, 1, 0], pool[:, 1, 1] = 1.0, 2.0
    c = mb.Cache(pool, torch.zeros(2, cols, dtype=torch.int32, device=DEV), ints([2 ** 31 - 20, 5]), ints([cols, 1]))
    c.table[1, 0] = 1
    q = randn(gen(4), 2, 1, 64, typ=torch.float16)
    out = c.attend(q, ints([0, 1]), 0)
    c.check()
    assert bool((out[0] == 1).all()) and bool((out[1] == 2).all())


def test_a_fork_takes_its_window_whole_or_not_at_all(mb):
    c = mb.Cache.empty(1, 4, 1, 4, 8, 2, 2)
    one, keep = ints([0]), ints([[0]])
    for args in ((keep,), (keep, one), (keep, None, one), (None, one, one), (one, one, one)):
        with pytest.raises(ValueError):
            c.fork(one, ints([1]), *args)


def test_append_reports_bad_slots_and_skips_them(mb):
    cache = mb.Cache.empty(1, 2, 1, 4, 8, 2, 2)
    cache.pool.fill_(5.0)
    plan = mb.Rope(8, [], n_axes=1)
    x = torch.arange(5 * 8, device=DEV).reshape(5, 1, 8).to(torch.bfloat16)
    qo = torch.full_like(x, 9.0)
    pos = torch.zeros(1, 5, dtype=torch.int32, device=DEV)
    plan.append(x, x, x + 1, pos, cache, 0, ints([3, -1, 8, -2, 4]), q_out=qo)
    assert cache.status() == mb.MAP_EINTERNAL and cache.status() == mb.MAP_OK
    assert torch.equal(qo[[0, 4]], x[[0, 4]]) and bool((qo[1:4] == 9).all())
    assert torch.equal(cache.pool[0, 0, 0, 0, 3], x[0, 0]) and torch.equal(cache.pool[0, 1, 1, 0, 0], x[4, 0] + 1)
    assert int((cache.pool != 5).any(-1).sum()) == 4
    plan.append(None, x, x, pos, cache, 0, ints([0, 1, 2, 3, 4]))           # keys and values alone
    assert torch.equal(cache.pool[0, 1, 0, 0], x[:4, 0])


def test_page_calls_whose_shared_memory_is_48_kb(mb):
    """Entries and sequences that take just under 48 KB beside the kernels' fixed words, in a new process, where no larger
    call came before."""
    prog = """
import torch
from paper_2608_06411_gb300 import binding as mb
i32 = dict(dtype=torch.int32, device="cuda")
for seqs in (72192, 73152, 73184):
    c = mb.Cache.empty(1, 2000, 1, 4, 8, seqs, 1)
    who = torch.arange(2000, **i32)
    assert c.extend(who).tolist() == [4 * i for i in range(2000)]
    c.free(who)
    c.extend(who[:1000])
    c.fork(torch.arange(2000, **i32) % 1000, torch.arange(3000, 5000, **i32), torch.zeros(2000, 0, **i32),
           torch.zeros(2000, **i32), torch.ones(2000, **i32))
    c.check()
    assert c.length[:5000].sum().item() == 1000
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", prog], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# ----------------------------------------------------------------------------- attention

def filled(mb, typ, dh, hk, page, lens, seed, layers=1, spare=2, extra_seqs=0):
    """A cache whose sequences have the given lengths, pages at random places, NaN wherever no row is."""
    g = gen(seed)
    used = [-(-t // page) for t in lens]
    pages, max_pages = sum(used) + spare, max([1] + used)
    cache = mb.Cache.empty(layers, pages, hk, page, dh, len(lens) + extra_seqs, max_pages, typ)
    cache.pool.fill_(float("nan"))
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = 0
    for s, (n, t) in enumerate(zip(used, lens)):
        mine = order[at: at + n]
        cache.table[s, :n] = mine
        cache.refs[mine.long()] = 1
        at += n
        if t:
            i = torch.arange(t, device=DEV)
            for l in range(layers):
                for kv in (0, 1):
                    cache.pool[l, kv][mine[i // page].long(), :, i % page] = randn(g, t, hk, dh, typ=typ)
    cache.length[: len(lens)] = ints(lens)
    return cache


def check_attend(got, q, cache, layer, seqs, scale, typ):
    """Scores: tensor-core sums lose up to an ulp (2^-23) of their magnitude per 16 terms, plus the product with scale:
    dz = (dh / 16 + 3) 2^-23 of sum |q k| scale; exp turns that into a relative error of p, twice (p and their sum),
    with 2^-21 for exp2 and its argument (|z| up to 40: 40 * 2^-24).  p as two halves of the cache's type keeps 2^-16;
    the sum over n rows loses an ulp per 16, and a few joins of parts."""
    table, lens = cache.table.cpu().tolist(), cache.length.cpu().tolist()
    page = cache.page
    for i, s in enumerate(seqs):
        if s < 0:
            continue
        slots = [table[s][t // page] * page + t % page for t in range(lens[s])]
        k, v = (f64(rows_of(cache.pool[layer: layer + 1], slots))[0, j] for j in (0, 1)) if slots else \
            (np.zeros((0, cache.heads, cache.dh)),) * 2
        want, mag, dz = H.attend(f64(q[i]), k, v, scale)
        e = 2 * (cache.dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + 2.0 ** -16 + (len(slots) / 16 + 64) * 2.0 ** -23
        tol = half_step(typ) * np.abs(want) * 1.001 + e * mag + tiny(typ)
        off = np.abs(f64(got[i]) - want)
        assert (off <= tol).all(), (i, float((off / np.maximum(tol, 1e-30)).max()))


ATTENDS = [
    # type, dh, hk, group, page, lens
    ("bf16", 128, 2, 4, 16, [0, 1, 15, 16, 17, 63, 64, 65, 300]),
    ("f16", 64, 1, 1, 16, [5, 0, 1000]),
    ("bf16", 80, 3, 2, 8, [33, 129, 2]),
    ("f16", 96, 2, 8, 32, [200, 31]),
    ("bf16", 192, 1, 3, 64, [1, 700]),
    ("f16", 256, 2, 2, 16, [129, 64, 2000]),
    ("bf16", 128, 1, 16, 5, [77, 13, 0]),
    ("bf16", 64, 1, 40, 1, [50, 3]),
    ("f16", 128, 4, 7, 48, [9000]),
    ("bf16", 128, 8, 4, 16, [200 + 37 * i for i in range(40)]),
    ("bf16", 64, 2, 17, 1024, [1500, 1023, 1024, 1025]),
    ("f16", 128, 1, 1, 3, [2, 1] * 150),
]


@pytest.mark.parametrize("case", ATTENDS, ids=["-".join(str(v) for v in c[:5]) for c in ATTENDS])
def test_attend_matches_the_formula(mb, case):
    typ, dh, hk, group, page, lens = case
    typ = TYPES[typ]
    cache = filled(mb, typ, dh, hk, page, lens, 5, layers=2)
    seqs = list(range(len(lens) - 1, -1, -1)) + [-1, 0]
    q = randn(gen(6), len(seqs), hk * group, dh, typ=typ) * 1.5
    out = torch.full_like(q, 3.0)
    cache.attend(q, ints(seqs), 1, out=out)
    check_attend(out, q, cache, 1, seqs, dh ** -0.5, typ)
    assert bool((out[len(lens)] == 3.0).all())                       # the padding row
    for i, s in enumerate(seqs):
        assert s < 0 or lens[s] or bool((out[i] == 0).all())         # an empty sequence
    assert torch.equal(cache.attend(q, ints(seqs), 1, out=torch.full_like(q, 3.0)), out)      # repeatable
    (qv, _), (ov, base) = place(q, "packed"), place(torch.full_like(q, 7.0), "packed")
    cache.attend(qv, ints(seqs), 1, out=ov)
    ok = [i for i, s in enumerate(seqs) if s >= 0]
    assert torch.equal(ov[ok], out[ok])
    ov.fill_(7.0)
    assert bool((base == 7.0).all())
    cache.check()


def test_attend_values_at_the_edges(mb):
    cache = filled(mb, torch.bfloat16, 64, 1, 16, [100, 3, 40], 2)
    q = randn(gen(1), 3, 2, 64, typ=torch.bfloat16)
    out = cache.attend(q, ints([0, 1, 2]), 0, scale=0.0)             # equal weights: the mean
    check_attend(out, q, cache, 0, [0, 1, 2], 0.0, torch.bfloat16)
    out = cache.attend(q, ints([0, 1, 2]), 0, scale=-0.125)
    check_attend(out, q, cache, 0, [0, 1, 2], -0.125, torch.bfloat16)
    out = cache.attend(q * 1e4, ints([0, 1, 2]), 0)                  # one row takes all
    assert bool(torch.isfinite(out).all())
    cache.pool[0, 1][cache.table[1, 0].long(), 0, 1] = float("inf")  # an infinite value: sequence 1 alone has it
    out = cache.attend(q, ints([0, 1, 2]), 0)
    assert bool(torch.isinf(out[1]).all()) and bool(torch.isfinite(out[[0, 2]]).all())
    cache.pool[0, 0][cache.table[2, 0].long(), 0, 7] = float("nan")  # a visible NaN key
    out = cache.attend(q, ints([0, 1, 2]), 0)
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isfinite(out[0]).all())
    out = torch.full_like(q, 4.0)
    cache.attend(q, ints([5, 0, -3]), 0, out=out)
    assert cache.status() == mb.MAP_EINTERNAL and bool((out[[0, 2]] == 4.0).all()) and bool(torch.isfinite(out[1]).all())
    with pytest.raises(ValueError):
        cache.attend(q.half(), ints([0, 1, 2]), 0)
    with pytest.raises(mb.MapError):
        cache.attend(q, ints([0, 1, 2]), 1)
    assert cache.attend(q[:0], ints([]), 0).shape == (0, 2, 64)


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_infinite_values_of_small_weights(mb, typ):
    """Weights from 1 down to 2^-110 (scores 8 k, in 1 / ln 2 steps): an infinite value of any of them is infinite in the
    sum.  Scores of minus infinity alone give no weights: NaN."""
    typ = TYPES[typ]
    for gap in (1.0, 3.0, 5.0, 9.5):                                  # 11, 34, 57 and 109 powers of two
        for sign, row in ((1.0, 5), (-1.0, 69)):                      # of the first warp in both tiles
            cache = filled(mb, typ, 64, 1, 16, [100, 40], 2)
            page = cache.table[0, row // 16].long()
            keys, values = cache.pool[0, 0, :, 0], cache.pool[0, 1, :, 0]
            keys[cache.table[0, :7].long()] = 0.0
            keys[cache.table[0, 0].long(), 3] = gap
            values[page, 5, 7] = sign * float("inf")
            q = torch.ones(2, 2, 64, dtype=typ, device=DEV)
            out = cache.attend(q, ints([0, 1]), 0)
            assert bool((out[0, :, 7] == sign * float("inf")).all()), (gap, out[0, :, 7])
            out[0, :, 7] = 0.0
            assert bool(torch.isfinite(out).all())
    keys[cache.table[0, :7].long(), :, 0] = float("-inf")
    out = cache.attend(q, ints([0, 1]), 0)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isfinite(out[1]).all())


def test_pool_offsets_past_32_bits(mb):
    """The last pages of a pool of 2^33 bytes: appended, attended, forked and freed."""
    dh, hk, page = 128, 8, 64
    pages = (1 << 32) // (4 * hk * page * dh) + 3                    # 2 layers, K and V: over 2^32 elements
    cache = mb.Cache.empty(2, pages, hk, page, dh, 3, 4)
    cache.refs[: pages - 3] = 1                                      # the free pages are the last
    plan = mb.Rope(dh, [1.0] * 64)
    g = gen(4)
    k, v, q = (randn(g, 70, h, dh, typ=torch.bfloat16) for h in (hk, hk, 16))
    slots = cache.extend(ints([0]), ints([70]), rows=70)
    pos = torch.arange(70, dtype=torch.int32, device=DEV)[None]
    plan.append(q, k, v, pos, cache, 1, slots)
    rk = plan.rotate(None, k, pos)[1]
    cache.fork(ints([0]), ints([1]))
    cache.check()
    assert cache.table[1, :2].cpu().tolist() == [pages - 3, pages - 1]
    for s in (0, 1):
        at = cache.table[s, :2].cpu().tolist()
        sl = [at[t // page] * page + t % page for t in range(70)]
        got = rows_of(cache.pool[1:], sl)[0]
        assert torch.equal(got[0], rk) and torch.equal(got[1], v)
    out = cache.attend(q[:2], ints([1, 0]), 1)
    check_attend(out, q[:2], cache, 1, [1, 0], dh ** -0.5, torch.bfloat16)


# ----------------------------------------------------------------------------- streams, graphs, the whole path

def test_calls_on_a_stream_of_the_callers(mb):
    case = ROTATIONS[0]
    typ, q, k, wq, wk, pos, inv, ax, plan = rotation(mb, case)
    cache = filled(mb, typ, 128, 4, 16, [40, 20], 3)
    want = plan.rotate(q, k, pos, wq, wk)
    wgrad = plan.grad(q, k, pos, q, k, wq, wk)
    watt = cache.attend(q.expand(2, -1, -1), ints([0, 1]), 0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = plan.rotate(q, k, pos, wq, wk, stream=s)
    ggrad = plan.grad(q, k, pos, q, k, wq, wk, stream=s)
    gatt = cache.attend(q.expand(2, -1, -1), ints([0, 1]), 0, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*want, *wgrad, watt), (*got, *ggrad, gatt)))


def test_a_dropped_cache_waits_for_every_stream(mb):
    """The same of the pages that Cache.empty made: rows appended on another stream land before they are handed out."""
    cache = mb.Cache.empty(1, 64, 2, 16, 64, 2, 32, dtype=torch.float16)
    plan, x = mb.Rope(64, [1.0]), torch.ones(300, 2, 64, dtype=torch.float16, device=DEV)
    pos, slots = torch.zeros(1, 300, dtype=torch.int32, device=DEV), cache.extend(ints([0]), ints([300]), rows=300)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)
        plan.append(None, x, x, pos, cache, 0, slots)
    place, size = cache.pool.data_ptr(), cache.pool.numel()
    del cache
    other = torch.full((size,), 7.0, dtype=torch.float16, device=DEV)
    assert other.data_ptr() != place
    torch.cuda.synchronize()
    assert bool((other == 7).all())


def test_append_of_rows_at_any_alignment(mb):
    """Half of 72 columns turned, 18 pairs, and heads that begin on odd elements: keys and values reach their slots."""
    rows, hq, hk, dh = 45, 6, 3, 72
    case = ("bf16", rows, hq, hk, dh, 36, 2, False, True, "odd", 5000)
    typ, q, k, wq, wk, pos, inv, ax, plan = rotation(mb, case)
    v = randn(gen(8), rows, hk, dh, typ=typ)
    cache = mb.Cache.empty(1, 4, hk, 16, dh, 2, 3)
    cache.pool.fill_(5.0)
    slots = cache.extend(ints([1]), ints([rows]), rows=rows)
    slots[7] = -1
    (qv, _), (kv, _), (vv, _) = (place(t, "odd") for t in (q, k, v))
    qo = torch.full_like(q, 7.0)
    plan.append(qv, kv, vv, pos, cache, 0, slots, wq, wk, q_out=qo)
    cache.check()
    got = cache.pool[0].transpose(2, 3).reshape(2, 64, hk, dh)        # by slot
    on = [r for r in range(rows) if r != 7]
    at = slots[on].long()
    check_rotated(qo[on], q[on], wq, pos[:, on], inv, ax, False, typ)
    check_rotated(got[0][at], k[on], wk, pos[:, on], inv, ax, False, typ)
    assert torch.equal(got[1][at], v[on])
    rest = torch.ones(64, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert bool((got[:, rest] == 5).all()) and bool((qo[7] == 7).all())


def test_a_cache_dropped_while_another_stream_attends(mb):
    """Attention's scratch is not handed out again before the stream that uses it is done."""
    cache = filled(mb, torch.float16, 64, 2, 16, [300, 20], 3)
    q = randn(gen(5), 2, 8, 64, typ=torch.float16)
    seqs = ints([0, 1])
    want = cache.attend(q, seqs, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)                               # some 50 ms
        got = cache.attend(q, seqs, 0)
    place, size, keep = cache._ws.data_ptr(), cache._ws.numel(), (cache.pool, cache.table, cache.length, cache.refs, cache.status_word)
    del cache
    other = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    assert other.data_ptr() != place
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(keep) == 5


def test_inputs_dropped_while_the_given_stream_reads_them(mb):
    """`stream=` calls on temporaries: their memory is not handed out before that stream is done with it."""
    s, g = torch.cuda.Stream(), gen(7)
    plan, ctx = mb.Rope(64, [0.5 ** i for i in range(32)]), handoff_context(mb, 512)
    q, k, dy = (randn(g, 3000, h, 64, typ=torch.bfloat16) for h in (4, 2, 4))
    pos = torch.randint(0, 900, (1, 3000), generator=g, device=DEV, dtype=torch.int32)
    w = torch.ones(64, device=DEV, dtype=torch.bfloat16)
    vis = torch.randint(0, 999, (1, 2000, 512), generator=g, device=DEV, dtype=torch.int16)
    text, keep = vis[0, :100].clone(), torch.arange(0, 2000, 2, dtype=torch.int32, device=DEV)[None]

    def fresh():
        c = filled(mb, torch.bfloat16, 64, 2, 16, [40, 0, 0], 3, spare=400)
        wide = torch.zeros(3, 200, dtype=torch.int32, device=DEV)
        wide[:, : c.table.shape[1]] = c.table
        return mb.Cache(c.pool, wide, c.length, c.refs)

    def calls(c, x, stream):
        """Every call, on tensors of the dict x."""
        out = list(plan.rotate(x["q"], x["k"], x["pos"], x["w"], x["w"], stream=stream))
        out += plan.grad(x["dy"], None, x["pos"], x["q"], None, x["w"], stream=stream)[::2]
        out += ctx.assemble_axes(x["vis"], x["keep"], x["text"], [100], [(1, 40, 50)], stream=stream)
        slots = c.extend(x["seqs"], x["counts"], rows=3000, stream=stream)
        out.append(plan.append(x["q"], x["k"], x["k"], x["pos"], c, 0, slots, x["w"], x["w"], stream=stream))
        c.fork(x["one"], x["two"], x["kept"], x["base"], x["span"], stream=stream)
        out.append(c.attend(x["q"][:2], x["both"], 0, stream=stream))
        c.free(x["one"], stream=stream)
        return out

    values = dict(q=q, k=k, dy=dy, pos=pos, w=w, vis=vis, text=text, keep=keep, seqs=ints([1]), counts=ints([3000]), one=ints([1]),
                  two=ints([2]), kept=ints([[7, 9, 2000]]), base=ints([3]), span=ints([2990]), both=ints([0, 2]))
    a, b = fresh(), fresh()
    want = calls(a, values, None)
    torch.cuda.synchronize()
    temps = {n: t.clone() for n, t in values.items()}
    at, sizes = {t.data_ptr() for t in temps.values()}, [(t.shape, t.dtype) for t in temps.values()]
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)                               # some 50 ms
    got = calls(b, temps, s)
    del temps
    others = [torch.full(shape, 1, dtype=typ, device=DEV) for shape, typ in sizes]
    assert not at & {t.data_ptr() for t in others}
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want, strict=True))
    for c in (a, b):
        c.check()
    assert all(torch.equal(x, y) for x, y in ((a.table, b.table), (a.length, b.length), (a.refs, b.refs)))


def test_assemble_axes_on_a_stream_and_its_refusals(mb):
    ctx = handoff_context(mb, 512)
    vis, text = torch.ones((1, 8, 512), dtype=torch.int16, device=DEV), torch.full((2, 512), 2, dtype=torch.int16, device=DEV)
    keep, grid = ints([[1, 7]]), [(2, 2, 2)]
    want = ctx.assemble_axes(vis, keep, text, [2], grid)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = ctx.assemble_axes(vis, keep, text, [2], grid, stream=s)
    held = ctx.assemble_axes(vis, keep, text, [2], grid, seq=torch.zeros_like(want[0]), stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + want, got + held))
    for bad in (dict(keep=keep.cpu()), dict(keep=keep.long()), dict(text=text.cpu()), dict(text=text.to(torch.uint8)),
                dict(seq=torch.zeros(4, 512, dtype=torch.uint8, device=DEV)), dict(seq=torch.zeros(4, 512, dtype=torch.int16)),
                dict(pos=torch.zeros(3, 4, dtype=torch.int32))):
        with pytest.raises(ValueError):
            ctx.assemble_axes(**{**dict(vis=vis, keep=keep, text=text, lens=[2], grids=grid), **bad})


def test_a_decoding_step_captured_and_replayed(mb):
    """extend, append and attend of a padded batch in one graph, replayed with new rows and another set of sequences."""
    dh, hk, hq, n = 64, 2, 8, 4
    caches = [filled(mb, torch.float16, dh, hk, 16, [30, 0, 15, 16, 47], 8, spare=30) for _ in range(2)]
    for c in caches:                                                 # room for longer rows
        wide = torch.zeros(5, 9, dtype=torch.int32, device=DEV)
        wide[:, : c.table.shape[1]] = c.table
        c.__init__(c.pool, wide, c.length, c.refs)
    plan = mb.Rope(dh, [0.9 ** i for i in range(32)])
    seqs = ints([0, 1, 2, -1])
    q, k, v = (randn(gen(1), n, h, dh, typ=torch.float16) for h in (hq, hk, hk))
    pos = ints([[30, 0, 15, 0]])
    out = torch.full((n, hq, dh), 3.0, dtype=torch.float16, device=DEV)

    def step(c, out):
        slots = c.extend(seqs)
        qr = plan.append(q, k, v, pos, c, 0, slots)
        c.attend(qr, seqs, 0, out=out)

    want = [out.clone() for _ in range(3)]
    inputs = [(ints([0, 1, 2, -1]), 1), (ints([4, -1, 0, 1]), 2), (ints([0, 1, 2, 3]), 3)]

    def feed(i):
        seqs.copy_(inputs[i][0])
        for t, h in ((q, hq), (k, hk), (v, hk)):
            t.copy_(randn(gen(10 * inputs[i][1] + h), n, h, dh, typ=torch.float16))

    for i in range(3):
        feed(i)
        step(caches[0], want[i])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=warm):
        step(caches[1], out)
    for i in range(3):
        feed(i)
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), i
    assert torch.equal(caches[0].length, caches[1].length) and torch.equal(caches[0].refs, caches[1].refs)
    caches[1].check()


def test_gradient_captured_and_replayed_beside_an_eager_one(mb):
    typ, q, k, wq, wk, pos, inv, ax, plan = rotation(mb, ROTATIONS[15])
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    g = torch.cuda.CUDAGraph()
    plan.grad(dq, dk, pos, q, k, wq, wk)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        held = plan.grad(dq, dk, pos, q, k, wq, wk)
    for seed in (1, 2):
        dq.copy_(randn(gen(seed), *dq.shape, typ=typ))
        g.replay()
        eager = plan.grad(dq, dk, pos, q, k, wq, wk)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def test_an_image_answered_twice_from_one_cache(mb):
    """The whole path: score, select and assemble an image's tokens; its full prompt and two questions, each with its own
    kept tokens, in one cache; every layer's pages hold what the pruned prompt alone would give, and attention over
    the fork is attention over those rows."""
    from paper_2608_06411_gb300 import workloads as W
    dims = W.PredictorDims(D=512, Dh=256, dp=64)
    w = W.make_weights(dims, seed=7)
    wl = W.WORKLOADS["c0"]
    grid, K, dh, hk, hq, page = (2, 10, 12), 31, 64, 2, 8, 16
    N = grid[0] * grid[1] * grid[2]
    vis = np.stack([W.make_image(wl, 0, N=N, D=512)] * 2)
    lens = np.array([5, 9], np.int32)
    text = np.concatenate([W.make_text(wl, b, int(lens[b]), D=512) for b in range(2)])
    ctx = mb.Context({k: torch.from_numpy(v.view(np.int16)).to(DEV) for k, v in w.items()}, 512, 256, 64)
    vis_t, text_t = (torch.from_numpy(a.view(np.int16)).to(DEV) for a in (vis, text))
    keep, _ = ctx.select(ctx.score(text_t, vis_t, lens), vis_t, K)
    head = 7                                                         # rows of a system prompt before the image
    seq, pos = ctx.assemble_axes(vis_t, keep, text_t, lens, [grid] * 2, t_step=[2, 2], pos_offset=head)
    whole = torch.arange(N, dtype=torch.int32, device=DEV)[None]
    full, fpos = ctx.assemble_axes(vis_t[:1], whole, text_t[:1], [0], [grid], t_step=[2], pos_offset=head)
    ctx.check()
    # one layer's projection, and the system prompt's rows
    g = gen(2)
    proj = torch.randn(512, (hq + 2 * hk) * dh, generator=g, device=DEV) / 512 ** 0.5
    sys_rows = torch.randn(head, 512, generator=g, device=DEV)
    rows = torch.cat((sys_rows, full.view(torch.bfloat16).float()))
    rpos = torch.cat((torch.arange(head, dtype=torch.int32, device=DEV).expand(3, -1), fpos), 1).contiguous()
    wq, wk = ((1 + 0.1 * torch.randn(dh, generator=g, device=DEV)).bfloat16() for _ in range(2))
    inv = [10000.0 ** (-2.0 * i / dh) for i in range(dh // 2)]
    ax = [i % 3 for i in range(dh // 2)]
    plan = mb.Rope(dh, inv, axis=ax)
    cache = mb.Cache.empty(1, 64, hk, page, dh, 4, 24)

    def heads(x):
        y = (x @ proj).bfloat16()
        return y[:, : hq * dh].unflatten(1, (hq, dh)), y[:, hq * dh: -hk * dh].unflatten(1, (hk, dh)), \
            y[:, -hk * dh:].unflatten(1, (hk, dh))

    q, k, v = heads(rows)
    slots = cache.extend(ints([3]), ints([len(rows)]), rows=len(rows))
    plan.append(q, k, v, rpos, cache, 0, slots, wq, wk)
    cache.fork(ints([3, 3]), ints([0, 1]), keep, ints([head] * 2), ints([N] * 2))
    at = 0
    for b in range(2):                                               # the question's rows behind the kept ones
        m = int(lens[b])
        ids = pos[:, at + K: at + K + m].contiguous()
        tq, tk, tv = heads(seq[at + K: at + K + m].view(torch.bfloat16).float())
        s = cache.extend(ints([b]), ints([m]), rows=m)
        tq = plan.append(tq, tk, tv, ids, cache, 0, s, wq, wk)
        out = cache.attend(tq[-1:], ints([b]), 0)
        cache.check()
        # the same from the definition, in 64 bits
        kept = keep[b].long()
        kk = torch.cat((k[:head], k[head + kept], tk)).double().cpu().numpy()
        vv = torch.cat((v[:head], v[head + kept], tv)).double().cpu().numpy()
        kpos = torch.cat((rpos[:, :head], pos[:, at: at + K + m]), 1).cpu().numpy()
        ref, _ = H.rotate(kk, f64(wk), kpos, inv, ax, False, 1e-6)
        sl = [int(x) for t in range(-(-(head + K + m) // page)) for x in [cache.table[b, t]]]
        sl = [sl[t // page] * page + t % page for t in range(head + K + m)]
        got = rows_of(cache.pool, sl)[0]
        assert np.abs(f64(got[0]) - ref).max() <= 2 ** -8 * np.abs(ref).max() and (f64(got[1]) == vv).all()
        check_attend(out, tq[-1:], cache, 0, [b], dh ** -0.5, torch.bfloat16)
        at += K + m
    assert cache.length.cpu().tolist() == [head + K + 5, head + K + 9, 0, head + N]
    cache.free(ints([0, 1, 3]))
    assert int(cache.refs.sum()) == 0
    ctx.close()


# ----------------------------------------------------------------------------- calls from several host threads

def together(calls, times=30000):
    """Codes other than 0 that the calls returned, each made over and over by a host thread of its own."""
    codes = []

    def work(call):
        for _ in range(times):
            rc = call()
            if rc:
                codes.append(rc)

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return codes


@pytest.mark.parametrize("dh,groups", [(64, (16, 1)), (128, (8, 1)), (256, (16, 1))])
def test_attend_of_two_caches_from_two_threads(mb, dh, groups):
    """Groups of more and of fewer query heads, and so launches of one kernel with more and with less shared memory."""
    seqs, calls, held = ints([0, 1]), [], []
    for g in groups * 2:
        c, st = filled(mb, torch.float16, dh, 1, 16, [40, 20], 3), torch.cuda.Stream()
        q = randn(gen(4), 2, g, dh, typ=torch.float16)
        out = torch.empty_like(q)
        held.append((c, q, out, c.attend(q, seqs, 0)))
        args = (c.desc, 0, mb._heads(q, 2, dh, q.dtype, q.device), seqs.data_ptr(), 2, dh ** -0.5,
                mb._heads(out, 2, dh, q.dtype, q.device), c._ws.data_ptr(), st.cuda_stream)
        calls.append(lambda args=args, st=st: mb.lib.map_cache_attend(*args))
    torch.cuda.synchronize()
    assert together(calls) == []
    assert all(torch.equal(out, want) for _, _, out, want in held)


@pytest.mark.parametrize("call", ["extend", "fork"])
def test_page_calls_of_two_caches_from_two_threads(mb, call):
    """4096 and 2500 entries at the same time, each on caches of their own.  (Children stay empty: their parents are.)"""
    calls, held = [], []
    for n in (4096, 2500) * 2:
        c, st = mb.Cache.empty(1, 16, 1, 4, 8, 2 * n, 1), torch.cuda.Stream()
        who, kids, slots, none = ints(list(range(n))), ints(list(range(n, 2 * n))), ints([0] * n), ints([0] * n)
        held.append((c, who, kids, slots, none, st))
        if call == "extend":
            args = (c.desc, who.data_ptr(), none.data_ptr(), n, n, slots.data_ptr(), st.cuda_stream)
            calls.append(lambda args=args: mb.lib.map_cache_extend(*args))
        else:
            args = (c.desc, who.data_ptr(), kids.data_ptr(), n, None, 0, None, None, st.cuda_stream)
            calls.append(lambda args=args: mb.lib.map_cache_fork(*args))
    torch.cuda.synchronize()
    assert together(calls, 10000) == []
    for c, *_ in held:
        c.check()


def test_select_of_two_contexts_from_two_threads(mb):
    """A context a thread, images of 2880 and of 300 tokens: the selection's launches differ in shared memory too."""
    from paper_2608_06411_gb300 import workloads as W
    w = {n: torch.from_numpy(v.view(np.int16)).to(DEV) for n, v in W.make_weights(W.PredictorDims(D=512, Dh=256, dp=64), seed=7).items()}
    calls, held = [], []
    for N, k in ((2880, 160), (300, 24)) * 2:
        ctx, st = mb.Context(w, 512, 256, 64), torch.cuda.Stream()
        vis, scores = randn(gen(N), 1, N, 512, typ=torch.bfloat16), torch.rand(1, N, generator=gen(1), device=DEV)
        keep = torch.zeros(1, k, dtype=torch.int32, device=DEV)
        held.append((ctx, vis, scores, keep, st, ctx.select(scores, vis, k)[0]))
        args = (ctx.h, scores.data_ptr(), vis.data_ptr(), 1, N, k, keep.data_ptr(), None, st.cuda_stream)
        calls.append(lambda args=args: mb.lib.map_select(*args))
    torch.cuda.synchronize()
    assert together(calls, 4000) == []
    for ctx, _, _, keep, _, want in held:
        assert ctx.status() == mb.MAP_OK and torch.equal(keep, want)
        ctx.close()
