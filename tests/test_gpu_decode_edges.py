"""Decoding over a shared and a bounded cache on the GPU where it can go wrong.

Tolerances as in test_gpu_decode.py, and: fp16's halves of a weight above zero are raised to 2^-24 of 2^15 each, so that a row adds
2^-38 of the base's weight at most (bf16: 2^-125, nothing beside the smallest numbers)."""
import math
import threading

import numpy as np
import pytest
import torch

from oracle import handoff_oracle as H
from test_gpu_decode import check, grouped, slots_of
from test_gpu_handoff import DEV, TYPES, f64, filled, gen, half_step, ints, mb, randn, rows_of, tiny  # noqa: F401

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


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_shared_of_values_without_weight(mb, typ):  # noqa: F811
    """An infinite value of a row whose weight is zero in fp32 is no number in the sum, as in map_cache_attend."""
    cache = grouped(mb, TYPES[typ], 64, 1, 16, [(320, [4, 9])], 2)
    cache.pool[0, 0] = torch.nan_to_num(cache.pool[0, 0]) * 0
    cache.pool[0, 0, cache.table[0, 0].long(), 0, 3, 0] = 1600.0     # a row that takes all, by 288 powers of two
    cache.pool[0, 1, cache.table[0, 2].long(), 0, 5, 7] = float("inf")
    q = torch.ones(2, 2, 64, dtype=TYPES[typ], device=DEV)
    for out in (cache.attend(q, ints([0, 1]), 0), cache.attend_shared(q, ints([0, 1]), 0, ints([0, 2]))):
        assert bool(torch.isnan(out[:, :, 7]).all())
        out[:, :, 7] = 0.0
        assert bool(torch.isfinite(out).all())


# ----------------------------------------------------------------------------- eviction: variants, refusals, replaced pages

def evicted(cache, weights, s, first, last, k):
    """Rows [layers, 2, rows, heads, dh] and weights [layers, heads, rows] that sequence s is to have afterwards."""
    slots = torch.tensor(slots_of(cache, s), device=DEV)
    n, layers, heads = len(slots), weights.shape[0], weights.shape[2]
    rows = cache.pool[:, :, slots // cache.page, :, slots % cache.page].permute(1, 2, 3, 0, 4)       # [layers, 2, heads, rows, dh]
    w = weights[:, s, :, :n]
    kept = w[..., first: n - last].sort(dim=-1, descending=True, stable=True).indices[..., :k].sort(dim=-1).values + first
    front, behind = (torch.arange(*r, device=DEV).expand(layers, heads, -1) for r in ((0, first), (n - last, n)))
    src = torch.cat((front, kept, behind), -1)
    return rows.gather(3, src[:, None, :, :, None].expand(-1, 2, -1, -1, rows.shape[-1])).transpose(2, 3), w.gather(-1, src)


VARIANTS = [
    # layers, heads, page, lens, first, last, k
    (38, 8, 16, [1000], 4, 100, 300), (38, 8, 16, [2000], 0, 0, 1500), (38, 8, 24, [3000], 35, 1, 700),
    (38, 8, 16, [4000], 1, 50, 2049), (38, 8, 5, [9000], 4, 9, 4000), (1, 2, 16, [70000], 35, 100, 30000),
    (2, 1, 64, [140001, 9], 0, 1, 100), (1, 1, 1024, [66000, 65000, 8193], 7, 0, 8100)]


@pytest.mark.parametrize("case", VARIANTS, ids=["-".join(str(v) for v in c) for c in VARIANTS])
def test_evict_of_every_number_of_candidates_a_thread(mb, case):  # noqa: F811
    """304 units a CTA each, with 4, 8, 13 and 16 candidates a thread and more than it holds; few units in clusters of eight CTAs, whose
    shares are looked at in several pieces.  Thousands of equal weights at the border."""
    layers, hk, page, lens, first, last, k = case
    cache = filled(mb, torch.float16, 8, hk, page, lens, 3, layers=layers)
    weights = torch.exp(2.5 * torch.randn(layers, len(lens), hk, cache.table.shape[1] * page, generator=gen(1), device=DEV))
    weights[:, :, hk // 2:] = (weights[:, :, hk // 2:] * 4).floor()
    was = [n if n - first - last <= k else first + k + last for n in lens]
    want = [evicted(cache, weights, s, first, last, k) if left < lens[s] else None for s, left in enumerate(was)]
    n = len(lens)
    cache.evict(weights, ints(range(n)), ints([first] * n), ints([last] * n), k)
    cache.check()
    assert cache.length.cpu().tolist() == was
    for s, left in enumerate(was):
        if want[s] is not None:
            assert torch.equal(rows_of(cache.pool, slots_of(cache, s)), want[s][0])
            assert torch.equal(weights[:, s, :, :left], want[s][1]) and bool((weights[:, s, :, left: lens[s]] == 0).all())


def test_evict_that_is_refused_leaves_the_table(mb):  # noqa: F811
    def refused(code, *args):
        state = [t.clone() for t in (cache.table, cache.length, cache.refs, cache.pool.view(torch.int16), weights)]
        cache.evict(weights, *args)
        assert cache.status() == code
        for a, b in zip(state, (cache.table, cache.length, cache.refs, cache.pool.view(torch.int16), weights)):
            assert torch.equal(a, b)

    cache = grouped(mb, torch.float16, 64, 1, 16, [(64, [5, 40]), (0, [100])], 1, spare=-2)          # two pages are free
    weights = torch.rand(1, 3, 1, cache.table.shape[1] * 16, generator=gen(1), device=DEV)
    refused(mb.MAP_ENOMEM, ints([0, 2]), None, None, 40)             # three shared pages to replace
    refused(mb.MAP_EINTERNAL, ints([0, 2, 0]), ints([32] * 3), None, 4)
    refused(mb.MAP_EINTERNAL, ints([0, 3]), ints([32] * 2), None, 4)
    refused(mb.MAP_EINTERNAL, ints([0, 2]), ints([32, -1]), None, 4)
    cache.length[2] = 1 << 20
    refused(mb.MAP_EINTERNAL, ints([0, 2]), ints([32, 0]), None, 4)
    cache.length[2] = 100
    for bad in (-1, cache.pool.shape[2]):
        good, cache.table[2, 5] = int(cache.table[2, 5]), bad
        refused(mb.MAP_EINTERNAL, ints([0, 2]), ints([32, 0]), None, 4)
        cache.table[2, 5] = good
    cache.evict(weights, ints([0, 2]), ints([32, 0]), None, 4)       # what was refused with them
    cache.check()
    assert cache.length.cpu().tolist() == [36, 104, 4]


def test_evict_replaces_the_shared_page_that_it_cuts(mb):  # noqa: F811
    """Nothing stays behind row 20: the shared page of rows 16 to 19 is replaced all the same, so that rows appended later
    are the sequence's own, and the call is refused where no page is free."""
    for spare in (-3, -4):                                           # one page free, none
        cache = grouped(mb, torch.float16, 64, 2, 16, [(64, [5, 40])], 1, spare=spare)
        weights = torch.rand(1, 2, 2, cache.table.shape[1] * 16, generator=gen(1), device=DEV)
        pages, rows = cache.table[0].clone(), rows_of(cache.pool, slots_of(cache, 0))
        other = rows_of(cache.pool, slots_of(cache, 1))
        cache.evict(weights, ints([0]), ints([20]), None, 0)
        if spare == -4:
            assert cache.status() == mb.MAP_ENOMEM and torch.equal(cache.table[0], pages) and int(cache.length[0]) == 69
            continue
        cache.check()
        assert int(cache.length[0]) == 20 and cache.table[0, 0] == pages[0] and cache.table[0, 1] != pages[1]
        assert cache.refs[pages[:5].long()].tolist() == [2, 1, 1, 1, 0] and int(cache.refs[cache.table[0, 1].long()]) == 1
        cache.pool[0, :, cache.table[0, 1].long(), :, 4:] = 9.0      # where rows behind come
        assert torch.equal(rows_of(cache.pool, slots_of(cache, 0)), rows[:, :, :20])
        assert torch.equal(rows_of(cache.pool, slots_of(cache, 1)), other)


# ----------------------------------------------------------------------------- together

def test_positions_go_on_after_an_eviction(mb):  # noqa: F811
    """Kept keys stay rotated by the positions they were appended with: the caller counts on from the tokens, not from the length."""
    dh, hk, hq, page, plan_freq = 64, 2, 4, 16, [0.9 ** i for i in range(32)]
    plan, cache = mb.Rope(dh, plan_freq), mb.Cache.empty(1, 8, hk, page, dh, 1, 5, torch.float16)
    weights = torch.zeros(1, 1, hk, 5 * page, device=DEV)
    one, first, last, budget, tokens = ints([0]), ints([4]), ints([8]), 20, 150
    raw = [randn(gen(i), tokens, h, dh, typ=torch.float16) for i, h in enumerate((hq, hk, hk))]
    token = torch.zeros(1, 1, dtype=torch.int32, device=DEV)         # positions: tokens so far, whatever has been evicted
    held = [[] for _ in range(hk)]                                   # tokens that a head holds
    for t in range(tokens):
        q, k, v = (x[t: t + 1] for x in raw)
        q = plan.append(q, k, v, token, cache, 0, cache.extend(one))
        out = cache.attend_weigh(q, one, 0, weights)
        token += 1
        for h in range(hk):
            held[h].append(t)
        n = len(held[0])
        assert n == int(cache.length[0])
        if n == 40:                                                  # back to first + budget + last
            for h in range(hk):
                kept = 4 + weights[0, 0, h, 4: n - 8].sort(descending=True, stable=True).indices[:budget].sort().values
                held[h] = held[h][:4] + [held[h][i] for i in kept.tolist()] + held[h][n - 8:]
            cache.evict(weights, one, first, last, budget)
    cache.check()
    assert int(cache.length[0]) < 40 < tokens
    for h in range(hk):
        pos = np.array([held[h]], dtype=np.int64)
        keys = H.rotate(f64(raw[1])[held[h]], None, pos, plan_freq, np.zeros(32, int), False, 0.0)[0][:, h: h + 1]
        want, mag, dz = H.attend(H.rotate(f64(raw[0])[-1:], None, np.array([[tokens - 1]]), plan_freq, np.zeros(32, int), False, 0.0)[0][0, 2 * h: 2 * h + 2],
                                 keys, f64(raw[2])[held[h]][:, h: h + 1], dh ** -0.5)
        # q and k are rotated and rounded once: 32 2^-24 and half a step each of the scores' products, which p has twice
        e = sums_error(dh, 40, dz) + 4.2 * half_step(torch.float16) * dz + 128 * 2.0 ** -24 * dz
        assert (np.abs(f64(out[0, 2 * h: 2 * h + 2]) - want) <= half_step(torch.float16) * np.abs(want) + e * mag + tiny(torch.float16)).all()


def test_evictions_of_several_caches_from_several_threads(mb):  # noqa: F811
    """Steps of rows appended, weighed and evicted, in caches whose calls take more and less shared memory than is had without asking:
    each cache ends as it does alone."""
    budget, steps, sets = 6, 150, []
    for n, dh, group in ((3000, 64, 16), (2, 64, 1), (3000, 256, 1), (2, 256, 2)):
        c = mb.Cache.empty(1, 4 * n, 1, 4, dh, n, 5, torch.float16)
        c.pool.normal_(generator=gen(n + dh))
        sets.append((n, c, randn(gen(dh), n, group, dh, typ=torch.float16), torch.cuda.Stream()))

    def work(n, c, q, weights, stream):
        seqs, first, last, counts = ints(range(n)), ints([1] * n), ints([2] * n), ints([3] * n)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for step in range(steps):
                c.extend(seqs, counts, rows=3 * n)
                c.attend_weigh(q, seqs, 0, weights)
                c.evict(weights, seqs, first, last, budget)
        stream.synchronize()

    results = []
    for threads in (False, True):
        copies, jobs = [], []
        for n, c, q, stream in sets:
            d = mb.Cache(*(t.clone() for t in (c.pool, c.table, c.length, c.refs)))
            w = torch.zeros(1, n, 1, 20, device=DEV)
            copies.append((d, w))
            jobs.append(threading.Thread(target=work, args=(n, d, q, w, stream)))
        torch.cuda.synchronize()
        for j in jobs:
            j.start()
            if not threads:
                j.join()
        for j in jobs:
            j.join()
        torch.cuda.synchronize()
        for d, _ in copies:
            d.check()
            assert bool((d.length == 1 + budget + 2).all())
        results.append([(d.pool.view(torch.int16), d.table, d.length, d.refs, w) for d, w in copies])
    for alone, beside in zip(*results):
        assert all(torch.equal(a, b) for a, b in zip(alone, beside))
        assert float(alone[-1].abs().sum()) > 0


def test_what_a_cache_remembers_of_its_calls_is_bounded(mb):  # noqa: F811
    cache = mb.Cache.empty(1, 8, 1, 4, 8, 2, 4)
    weights = torch.zeros(1, 2, 1, 16, device=DEV)
    for k in range(5000):
        cache.evict(weights, ints([-1]), None, None, k)
    cache.check()
    assert len(cache._sizes) <= 4096


def test_evict_refuses_a_k_that_no_int_holds(mb):  # noqa: F811
    cache = mb.Cache.empty(1, 8, 1, 4, 8, 1, 4)
    weights = torch.zeros(1, 1, 1, 16, device=DEV)
    cache.extend(ints([0]), ints([10]), rows=10)
    for k in (1 << 31, 1 << 32, (1 << 40) + 1):
        with pytest.raises(ValueError):
            cache.evict(weights, ints([0]), None, None, k)
    cache.evict(weights, ints([0]), None, None, (1 << 31) - 1)
    cache.check()
    assert int(cache.length[0]) == 10
