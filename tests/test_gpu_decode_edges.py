"""Decoding over a shared and a bounded cache on the GPU where it can go wrong.

Tolerances as in test_gpu_decode.py, and: fp16's halves of a weight above zero are raised to 2^-24 of 2^15 each, so that a row adds
2^-38 of the base's weight at most (bf16: 2^-125, nothing beside the smallest numbers)."""
import math

import pytest
import torch

from test_gpu_decode import check, grouped
from test_gpu_handoff import DEV, TYPES, gen, half_step, ints, mb, randn, tiny  # noqa: F401

pytestmark = pytest.mark.gpu


def sums_error(dh, n, dz):
    """Relative error of an output's sums over n rows whose scores have products that add up to dz (see test_gpu_decode.py)."""
    return 2 * (dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + 2.0 ** -16 + (n / 8 + n / 64 + 64) * 2.0 ** -23


@pytest.mark.parametrize("gap", [64, 200])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_shared_of_a_row_that_takes_all(mb, typ, gap):  # noqa: F811
    """A row of a small value takes all weight in front of 16000 large values of one sign, all of them in one CTA's run (250 tiles by
    304 heads for 304 CTAs).  Weights of 2^-64 are raised to 2^-38 at most, those of 2^-200 are zero in fp32."""
    typ, dh, hk, page, front, own = TYPES[typ], 64, 304, 16, 16000, 4
    whole, n = front // page, front + own
    cache = mb.Cache.empty(1, whole + 2, hk, page, dh, 2, whole + 1, typ)
    cache.table[:, :whole] = torch.arange(whole, dtype=torch.int32, device=DEV)
    cache.table[:, whole] = ints([whole, whole + 1])
    cache.refs[:] = ints([2] * whole + [1, 1])
    cache.length[:] = n
    cache.pool[0, 0], cache.pool[0, 1] = 0.0, 1000.0
    cache.pool[0, 0, 0, :, 5, 3] = gap * 8 * math.log(2)
    cache.pool[0, 1, 0, :, 5] = 0.001
    q = torch.ones(2, hk, dh, dtype=typ, device=DEV)
    dz = float(cache.pool[0, 0, 0, 0, 5, 3]) / 8
    w, v = math.exp(-dz), float(cache.pool[0, 1, 0, 0, 5, 0])
    want = (v + (n - 1) * 1000 * w) / (1 + (n - 1) * w)
    raised = (n - 1) * 1000 * (2.0 ** -38 if typ == torch.float16 else 2.0 ** -125) if gap < 126 else 0.0
    tol = half_step(typ) * (want + raised) + sums_error(dh, n, dz) * (want + raised) + raised + tiny(typ)
    for out in (cache.attend(q, ints([0, 1]), 0), cache.attend_shared(q, ints([0, 1]), 0, ints([0, 2]))):
        off = (out.double() - want).abs().max().item()
        assert off <= tol, (off, tol)
    cache.check()


LARGE = [("f16", 4, 1365), ("f16", 256, 1365), ("f16", 512, 1365), ("f16", 2048, 43680), ("f16", 8192, 43680),
         ("bf16", 256, 213), ("bf16", 1 << 28, 213 << 30)]


def large_scores(mb, typ, unit, key):  # noqa: F811
    """(cache, q, rows): four rows of each sequence have the same largest score by far: q's columns are 1, 3, 5 or 7 units, those
    rows' keys `key` (so that all sums are exact), other keys 1/64 of it at most, at random."""
    groups = [(1000, [9, 40, 3])]
    cache = grouped(mb, typ, 128, 2, 16, groups, 2)
    cache.pool[0, 0] = cache.pool[0, 0].clamp(-3, 3) * (key / 192)
    rows = [100, 900, 985, 995]                                      # the third in a tile of 32 rows, the last each sequence's own
    for s in range(3):
        for t in rows:
            cache.pool[0, 0, cache.table[s, t // 16].long(), :, t % 16] = key
    q = torch.ones(3, 8, 128, dtype=typ, device=DEV) * (torch.tensor([1.0, 3.0, 5.0, 7.0] * 2, device=DEV) * unit)[None, :, None].to(typ)
    return cache, q, rows


@pytest.mark.parametrize("case", LARGE, ids=["-".join(str(v) for v in c) for c in LARGE])
def test_attend_of_large_scores(mb, case):  # noqa: F811
    """Scores of 2^16 to 2^72 (in powers of two): what fp32 keeps of one is coarser than the weights' range, and equal scores have equal weights."""
    typ, unit, key = case
    typ = TYPES[typ]
    cache, q, rows = large_scores(mb, typ, unit, key)
    for out in (cache.attend(q, ints([0, 1, 2]), 0), cache.attend_shared(q, ints([0, 1, 2]), 0, ints([0, 3]))):
        for s in range(3):
            v = torch.stack([cache.pool[0, 1, cache.table[s, t // 16].long(), :, t % 16].double() for t in rows])
            want, mag = (x.mean(0).repeat_interleave(4, 0) for x in (v, v.abs()))
            tol = half_step(typ) * want.abs() * 1.001 + sums_error(128, 1040, 0.0) * mag + tiny(typ)
            off = (out[s].double() - want).abs()
            assert bool((off <= tol).all()), (s, float((off / tol).max()))
    cache.check()


@pytest.mark.parametrize("case", LARGE, ids=["-".join(str(v) for v in c) for c in LARGE])
def test_attend_weigh_of_large_scores(mb, case):  # noqa: F811
    """The same rows share the weight of each head between them."""
    typ, unit, key = case
    cache, q, rows = large_scores(mb, TYPES[typ], unit, key)
    weights = torch.zeros(1, 3, 2, cache.table.shape[1] * 16, device=DEV)
    out = cache.attend_weigh(q, ints([0, 1, 2]), 0, weights)
    assert torch.equal(out, cache.attend(q, ints([0, 1, 2]), 0))
    want = torch.zeros_like(weights)
    want[..., rows] = 1.0                                            # four heads, a quarter each
    off = float((weights - want).abs().max())
    assert off <= 2.0 ** -19 + (1040 / 16 + 64) * 2.0 ** -23, off
    cache.check()


# ----------------------------------------------------------------------------- lengths just below 2^31

def long_cache(mb, last, dh=8):  # noqa: F811
    """A cache of one sequence of 2^31 - 20 rows in pages of 16, all of them page 0 but the last `last`, which are 1, 2, ..."""
    cols = (1 << 27) - 1
    cache = mb.Cache.empty(1, last + 3, 1, 16, dh, 1, cols, torch.float16)
    cache.pool.normal_(generator=gen(3))
    cache.table[0, cols - last:] = torch.arange(1, last + 1, dtype=torch.int32, device=DEV)
    cache.length[0] = (1 << 31) - 20
    cache.refs[: last + 1] = 1
    return cache


def test_evict_at_lengths_just_below_32_bits(mb):  # noqa: F811
    """A window behind 2^31 - 720 rows: what lies in front of it, its pages' other rows among them, stays."""
    cache = long_cache(mb, 60)
    n, first, last, k = (1 << 31) - 20, (1 << 31) - 720, 100, 50
    before = cache.pool.clone()
    weights = torch.full((1, 1, 1, cache.table.shape[1] * 16), 3.0, device=DEV)
    weights[..., first: n] = torch.rand(n - first, generator=gen(1), device=DEV)
    was = weights[0, 0, 0, first: n].clone()
    cache.evict(weights, ints([0]), ints([first]), ints([last]), k)
    cache.check()
    left = first + k + last
    assert int(cache.length[0]) == left and bool((cache.refs[1: 61] == (torch.arange(60, device=DEV) < 26).int()).all())
    src = torch.cat((was[: n - first - last].sort(descending=True, stable=True).indices[:k].sort().values,
                     torch.arange(n - first - last, n - first, device=DEV)))
    w = weights[0, 0, 0]
    assert torch.equal(w[first: left], was[src]) and bool((w[left: n] == 0).all())
    assert bool((w[:first] == 3).all()) and bool((w[n:] == 3).all())
    # rows in the last 60 pages, in order
    rows, had = (p[0, :, 1: 61, 0].reshape(2, 960, 8) for p in (cache.pool, before))
    base = (1 << 31) - 16 - 960
    assert torch.equal(rows[:, first - base: left - base], had[:, src + first - base])
    assert torch.equal(rows[:, : first - base], had[:, : first - base]) and torch.equal(cache.pool[0, :, 0], before[0, :, 0])


def test_evict_of_all_rows_of_a_length_just_below_32_bits(mb):  # noqa: F811
    """All rows but five stay: every loop over rows goes almost to 2^31.  (Pages repeat, so that all rows are alike.)"""
    cache = long_cache(mb, 0)
    cache.pool.fill_(2.0)
    n, gone = (1 << 31) - 20, [10, 1000, 1 << 30, (1 << 31) - 23, (1 << 31) - 21]
    weights = torch.zeros(1, 1, 1, n + 4, device=DEV)
    w = weights[0, 0, 0]
    for at in range(0, n, 1 << 28):
        to = min(n, at + (1 << 28))
        w[at: to] = torch.arange(at, to, dtype=torch.int32, device=DEV) % 1021 + 1
    w[gone] = 0.0
    was = w.clone()
    cache.evict(weights, ints([0]), None, None, n - 5)
    cache.check()
    assert int(cache.length[0]) == n - 5 and cache.refs.cpu().tolist() == [1, 0, 0] and bool((cache.pool == 2).all())
    for i, (a, b) in enumerate(zip([-1] + gone, gone + [n])):
        assert torch.equal(w[a + 1 - i: b - i], was[a + 1: b]), i
    assert bool((w[n - 5:] == 0).all())


@pytest.mark.parametrize("page", [16, 24, 5])
def test_attend_shared_at_lengths_just_below_32_bits(mb, page):  # noqa: F811
    """Two sequences with all but their last pages in common: their own rows begin at no multiple of a tile, and the tile behind
    their last row passes 2^31.  The own rows take all weight."""
    cols = ((1 << 31) - 1) // page
    own = 160 // page
    n, front = cols * page - 4, (cols - own) * page
    assert front % 64 != 0 and front + (n - front + 63) // 64 * 64 >= 1 << 31
    cache = mb.Cache.empty(1, 2 * own + 2, 1, page, 64, 2, cols, torch.float16)
    cache.pool[0, 0], cache.pool[0, 1] = 0.0, 1.0
    cache.pool[0, 0, 1:, :, :, 0] = 1600.0
    cache.pool[0, 1, 1:] = randn(gen(2), 2 * own + 1, 1, page, 64, typ=torch.float16)
    for s in range(2):
        cache.table[s, cols - own:] = 1 + s * own + torch.arange(own, dtype=torch.int32, device=DEV)
    cache.length[:] = n
    q = torch.ones(2, 1, 64, dtype=torch.float16, device=DEV)
    out = cache.attend_shared(q, ints([0, 1]), 0, ints([0, 2]))
    cache.check()
    for s in range(2):
        v = cache.pool[0, 1, 1 + s * own: 1 + (s + 1) * own, 0].reshape(-1, 64)[: n - front].double()
        want, mag = v.mean(0), v.abs().mean(0)
        off = (out[s, 0].double() - want).abs()
        assert bool((off <= half_step(torch.float16) * want.abs() * 1.001 + sums_error(64, n - front, 200.0) * mag + tiny(torch.float16)).all()), s


# ----------------------------------------------------------------------------- many groups

def test_attend_shared_of_groups_of_which_few_share(mb):  # noqa: F811
    """60001 groups: the first, the second, one in the middle and the last one share rows, the others are single sequences of a row."""
    cache = grouped(mb, torch.bfloat16, 64, 2, 16, [(1000, [5, 40, 1]), (0, [1])], 2)
    groups = [[0, 1], [2, 0, 1]] + [[3]] * 29998 + [[1, 2]] + [[3]] * 29999 + [[0, 2]]
    seqs, starts = sum(groups, []), [0]
    for g in groups:
        starts.append(starts[-1] + len(g))
    q = randn(gen(1), 1, 4, 64, typ=torch.bfloat16).expand(len(seqs), -1, -1).contiguous()
    out = cache.attend_shared(q, ints(seqs), 0, ints(starts))
    cache.check()
    v = cache.pool[0, 1, cache.table[3, 0].long(), :, 0].repeat_interleave(2, 0)
    alone = torch.tensor(seqs, device=DEV) == 3
    assert bool((out[alone] == v).all())
    several = (~alone).nonzero()[:, 0]
    check(out[several], q[several], cache, 0, [seqs[i] for i in several.tolist()], 0.125, torch.bfloat16)
    assert torch.equal(cache.attend_shared(q, ints(seqs), 0, ints(starts)), out)
