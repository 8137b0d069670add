"""Decoding over a shared and a bounded cache on the GPU (attend_shared, attend_weigh, evict) against the 64-bit models of
oracle/handoff_oracle.py.

Tolerances.  Scores: tensor-core sums lose up to an ulp (2^-23) of their magnitude per 16 terms, and the product with scale one more:
dz = (dh / 16 + 3) 2^-23 of sum |q k| scale; exp turns that into a relative error of p, twice (p and their sum), with 2^-19 for exp2
and its argument (|z| up to 40 powers of two: 40 * 2^-24).  p as two halves of the cache's type keeps 2^-16.  The sum over n rows loses
an ulp per 16 of either half, and an ulp per 64 where a greater score scales what is there; 64 more for the parts that join.
A row's summed weight has the error of its p and of their sum, and 2^-23 for the additions."""
import numpy as np
import pytest
import torch

from oracle import handoff_oracle as H
from test_gpu_handoff import DEV, TYPES, f64, filled, gen, half_step, ints, mb, place, randn, rows_of, same_state, tiny, together  # noqa: F401

pytestmark = pytest.mark.gpu


def slots_of(cache, s):
    """Slots of a sequence's rows, by the cache's table."""
    table, n, page = cache.table[s].cpu().tolist(), int(cache.length[s]), cache.page
    return [table[t // page] * page + t % page for t in range(n)]


def sequence(cache, layer, s):
    """Keys and values [rows, heads, dh] of a sequence in 64 bits."""
    slots = slots_of(cache, s)
    return (f64(rows_of(cache.pool[layer: layer + 1], slots))[0, j] for j in (0, 1)) if slots else (np.zeros((0, cache.heads, cache.dh)),) * 2


def check(got, q, cache, layer, seqs, scale, typ):
    for i, s in enumerate(seqs):
        if s < 0:
            continue
        k, v = sequence(cache, layer, s)
        want, mag, dz = H.attend(f64(q[i]), k, v, scale)
        n = k.shape[0]
        e = 2 * (cache.dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + 2.0 ** -16 + (n / 8 + n / 64 + 64) * 2.0 ** -23
        tol = half_step(typ) * np.abs(want) * 1.001 + e * mag + tiny(typ)
        off = np.abs(f64(got[i]) - want)
        assert (off <= tol).all(), (i, float((off / np.maximum(tol, 1e-30)).max()))


def grouped(mb, typ, dh, hk, page, groups, seed, layers=1, spare=4, room=0):  # noqa: F811
    """A cache of groups (rows of the common beginning, [rows behind it of each member]): the whole pages of a beginning are held by
    all members, everything else by one; NaN wherever no row is.  room: further columns of a table row."""
    g = gen(seed)
    lens, held = [], []
    for front, own in groups:
        for t in own:
            lens.append(front + t)
            held.append(front // page)
    used = [-(-t // page) for t in lens]
    pages = sum(used) + spare
    cache = mb.Cache.empty(layers, pages, hk, page, dh, len(lens), max([1] + used) + room, typ)
    cache.pool.fill_(float("nan"))
    order, at, s = torch.randperm(pages, generator=g, device=DEV).to(torch.int32), 0, 0
    for front, own in groups:
        first = order[at: at + front // page]
        at += front // page
        for t in own:
            n = used[s] - held[s]
            mine = torch.cat((first, order[at: at + n]))
            at += n
            cache.table[s, : used[s]] = mine
            cache.refs.index_add_(0, mine.long(), torch.ones_like(mine))
            cache.length[s] = front + t
            s += 1
    for s, t in enumerate(lens):
        i = torch.arange(t, device=DEV)
        rows = cache.table[s].long()[i // page]
        for l in range(layers):
            for kv in (0, 1):
                cache.pool[l, kv][rows, :, i % page] = randn(g, t, hk, dh, typ=typ)
    return cache


def starts_of(groups, n=None):
    at = [0]
    for _, own in groups:
        at.append(at[-1] + len(own))
    return at


SHARED = [
    # type, dh, hk, query heads a key head, page, groups
    ("bf16", 128, 2, 4, 16, [(320, [0, 1, 15, 16, 17, 64, 65])]),
    ("bf16", 128, 1, 1, 16, [(64, [3, 5])]),
    ("f16", 64, 1, 1, 16, [(1000, [5, 0, 40]), (30, [2, 1]), (15, [1, 1]), (0, [7, 300])]),
    ("f16", 80, 3, 2, 8, [(129, [33, 4, 2]), (700, [1])]),
    ("bf16", 96, 2, 8, 24, [(200, [31] * 20), (25, [1, 2])]),
    ("bf16", 192, 1, 3, 64, [(700, [1, 64, 0]), (64, [0, 0])]),
    ("f16", 256, 2, 2, 16, [(2000, [129, 64]), (33, [5] * 40)]),
    ("bf16", 256, 1, 7, 100, [(901, [100, 99, 1])]),
    ("f16", 128, 1, 16, 5, [(77, [13, 0, 1, 9, 9, 9, 9, 9, 9])]),
    ("bf16", 64, 1, 40, 1, [(50, [3, 1, 4, 0])]),
    ("f16", 128, 4, 7, 48, [(9000, [1, 200, 37])]),
    ("bf16", 128, 8, 4, 16, [(1000 + 37 * i, [20 + i, 5, 33 * i]) for i in range(12)]),
    ("f16", 64, 2, 130, 1024, [(2100, [5, 1000])]),
    ("bf16", 128, 1, 4, 16, [(48 + i % 40, [1] * (1 + i % 3)) for i in range(400)]),
    ("bf16", 80, 2, 33, 16, [(3000, [40] * 9)]),
    ("f16", 64, 1, 1, 16, [(64, [1, 5] * 700), (130, [3] * 1100)]),
]


@pytest.mark.parametrize("case", SHARED, ids=["-".join(str(v) for v in c[:5]) for c in SHARED])
def test_attend_shared_matches_the_formula(mb, case):  # noqa: F811
    typ, dh, hk, group, page, groups = case
    typ = TYPES[typ]
    cache = grouped(mb, typ, dh, hk, page, groups, 5, layers=2)
    n = sum(len(own) for _, own in groups)
    seqs, starts = list(range(n)), starts_of(groups)
    q = randn(gen(6), n, hk * group, dh, typ=typ) * 1.5
    out = torch.full_like(q, 3.0)
    cache.attend_shared(q, ints(seqs), 1, ints(starts), out=out)
    check(out, q, cache, 1, seqs, dh ** -0.5, typ)
    assert torch.equal(cache.attend_shared(q, ints(seqs), 1, ints(starts)), out)             # repeatable
    # any groups are right: a padding row and a sequence twice in the first one, all in one, none
    order = [seqs[0], -1] + seqs + [seqs[-1]]
    q2 = randn(gen(7), len(order), hk * group, dh, typ=typ) * 1.5
    for st in ([0] + [s + 2 for s in starts[1:-1]] + [len(order)], [0, len(order)], [0, 0, len(order), len(order)], list(range(len(order) + 1))):
        got = torch.full_like(q2, 7.0)
        cache.attend_shared(q2, ints(order), 1, ints(st), out=got)
        check(got, q2, cache, 1, order, dh ** -0.5, typ)
        assert bool((got[1] == 7.0).all())
    (qv, _), (ov, base) = place(q, "packed"), place(torch.full_like(q, 7.0), "packed")
    cache.attend_shared(qv, ints(seqs), 1, ints(starts), out=ov)
    assert torch.equal(ov, out)
    ov.fill_(7.0)
    assert bool((base == 7.0).all())
    cache.check()


LONG = [
    # many tiles a CTA: type, dh, hk, query heads a key head, page, rows in front, rows of each member
    ("bf16", 128, 2, 4, 16, 60000, [5, 70]),
    ("f16", 128, 2, 4, 64, 50001, [1 + 3 * i for i in range(40)]),
    ("bf16", 64, 4, 7, 8, 40000, [9] * 30),
    ("f16", 96, 2, 3, 5, 31003, [2, 3]),
    ("bf16", 80, 2, 5, 7, 33333, [1] * 64),
    ("f16", 192, 1, 2, 32, 60000, [40, 1, 1]),
    ("bf16", 256, 1, 8, 16, 50000, [33] * 20),
]


@pytest.mark.parametrize("case", LONG, ids=["-".join(str(v) for v in c[:6]) for c in LONG])
def test_attend_shared_of_long_beginnings(mb, case):  # noqa: F811
    """As `check`, with the 64-bit values computed by torch."""
    typ, dh, hk, group, page, front, own = case
    typ, n, scale = TYPES[typ], len(own), dh ** -0.5
    cache = grouped(mb, typ, dh, hk, page, [(front, own)], 9)
    q = randn(gen(6), n, hk * group, dh, typ=typ) * 1.5
    q[:, 1] *= 3                                                     # a head whose largest score rises by far along the rows
    out = cache.attend_shared(q, ints(range(n)), 0, ints([0, n]))
    cache.check()
    for i in (0, n // 2, n - 1):
        slots = torch.tensor(slots_of(cache, i), device=DEV)
        k, v = (cache.pool[0, j][slots // page, :, slots % page].double().transpose(0, 1) for j in (0, 1))
        qi = q[i].double().view(hk, group, dh)
        p = torch.softmax(qi @ k.transpose(1, 2) * scale, -1)
        want, mag = p @ v, p @ v.abs()
        dz = float((qi.abs() @ k.abs().transpose(1, 2)).max()) * scale
        e = 2 * (dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + 2.0 ** -16 + (len(slots) / 8 + len(slots) / 64 + 64) * 2.0 ** -23
        off = (out[i].double().view_as(want) - want).abs()
        tol = half_step(typ) * want.abs() * 1.001 + e * mag + tiny(typ)
        assert bool((off <= tol).all()), (i, float((off / tol).max()))
    assert torch.equal(cache.attend_shared(q, ints(range(n)), 0, ints([0, n])), out)


def test_attend_shared_does_not_depend_on_padding(mb):  # noqa: F811
    """What lies in a padding entry's queries changes nothing, bit for bit; two graphs of calls on one cache replayed in turn."""
    cache = grouped(mb, torch.float16, 64, 2, 16, [(330, [1, 1, 1])], 4)
    seqs, starts, q = ints([0, -1, 1, 2]), ints([0, 4]), randn(gen(1), 4, 8, 64, typ=torch.float16)
    want, graphs = None, []
    for fill in (0.0, 100.0, float("nan"), float("inf")):
        q[1] = fill
        out = cache.attend_shared(q, seqs, 0, starts)
        want = out[[0, 2, 3]].clone() if want is None else want
        assert torch.equal(out[[0, 2, 3]], want)
    for _ in range(2):
        g, x = torch.cuda.CUDAGraph(), q.clone()
        with torch.cuda.graph(g):
            y = cache.attend_shared(x, seqs, 0, starts)
        graphs.append((g, x, y))
    for _ in range(3):
        for i, (g, x, y) in enumerate(graphs):
            x.copy_(q * (1.0 - 0.5 * i))
            g.replay()
        for i, (g, x, y) in enumerate(graphs):
            assert torch.equal(y[[0, 2, 3]], cache.attend_shared(x, seqs, 0, starts)[[0, 2, 3]])
    cache.check()


def test_attend_shared_of_empty_and_bad_entries(mb):  # noqa: F811
    cache = grouped(mb, torch.bfloat16, 64, 2, 16, [(100, [5, 9, 0]), (40, [1, 30])], 3)
    cache.free(ints([2]))                                            # an empty sequence in a group
    q = randn(gen(1), 6, 4, 64, typ=torch.bfloat16)
    seqs, starts = [0, 1, 2, 3, 4, 0], ints([0, 3, 6])
    out = cache.attend_shared(q, ints(seqs), 0, starts)
    check(out, q, cache, 0, seqs, 0.125, torch.bfloat16)
    assert bool((out[2] == 0).all())
    cache.check()
    for bad in ([0, 3, 5], [1, 3, 6], [0, 4, 3], [0, 7, 6], [0, -1, 6], [0, 3, 1 << 30]):
        out = cache.attend_shared(q, ints(seqs), 0, ints(bad))       # reported, and each for itself
        check(out, q, cache, 0, seqs, 0.125, torch.bfloat16)
        assert cache.status() == mb.MAP_EINTERNAL and cache.status() == mb.MAP_OK
    out = torch.full_like(q, 4.0)
    cache.attend_shared(q, ints([0, 5, 1, -3, 3, 4]), 0, starts, out=out)
    assert cache.status() == mb.MAP_EINTERNAL and bool((out[[1, 3]] == 4.0).all())
    check(out, q, cache, 0, [0, -1, 1, -1, 3, 4], 0.125, torch.bfloat16)
    cache.length[1] = 1 << 20                                        # a length that no row can hold: as if it were empty
    out = cache.attend_shared(q, ints(seqs), 0, starts)
    assert cache.status() == mb.MAP_EINTERNAL and bool((out[1] == 0).all())
    check(out, q, cache, 0, [0, -1, 2, 3, 4, 0], 0.125, torch.bfloat16)
    cache.length[1] = 109
    for page in (-1, cache.pool.shape[2], 1 << 30):                  # a shared page outside the pool reads as page 0
        cache.table[:2, 3] = page
        out = cache.attend_shared(q, ints(seqs), 0, starts)
        assert cache.status() == mb.MAP_EINTERNAL
        check(out, q, cache, 0, [-1, -1, 2, 3, 4, -1], 0.125, torch.bfloat16)
    with pytest.raises(ValueError):
        cache.attend_shared(q.half(), ints(seqs), 0, starts)
    with pytest.raises(ValueError):
        cache.attend_shared(q, ints(seqs), 0, starts.long())
    with pytest.raises(ValueError):
        cache.attend_shared(q[:2], ints(seqs), 0, starts)
    with pytest.raises(mb.MapError):
        cache.attend_shared(q, ints(seqs), 1, starts)
    with pytest.raises(mb.MapError):
        cache.attend_shared(q, ints(seqs), 0, starts[:1])
    assert cache.attend_shared(q[:0], ints([]), 0, ints([0, 0])).shape == (0, 4, 64)


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_shared_values_at_the_edges(mb, typ):  # noqa: F811
    typ = TYPES[typ]
    groups = [(300, [9, 40, 3]), (64, [1, 1])]
    seqs, starts = list(range(5)), ints(starts_of(groups))

    def fresh():
        return grouped(mb, typ, 64, 1, 16, groups, 2)
    cache, q = fresh(), randn(gen(1), 5, 2, 64, typ=typ)
    for scale in (0.0, -0.125, 4.0):                                 # equal weights: the mean; the other way round; few rows take all
        out = cache.attend_shared(q, ints(seqs), 0, starts, scale=scale)
        check(out, q, cache, 0, seqs, scale, typ)
    page = cache.table[0, 2].long()                                  # a page that three share
    for value in (float("inf"), float("nan")):
        cache = fresh()
        cache.pool[0, 1][page, 0, 1, 5] = value                      # an infinite value, or none, in one column
        out = cache.attend_shared(q, ints(seqs), 0, starts)
        hit = torch.isinf(out) if value == float("inf") else torch.isnan(out)
        assert bool(hit[:3, :, 5].all()) and int(hit.sum()) == 6 and bool(torch.isfinite(out[3:]).all())
        cache = fresh()
        cache.pool[0, 1][cache.table[1, 19].long(), 0, 2, 5] = value  # in a row that one sequence has
        out = cache.attend_shared(q, ints(seqs), 0, starts)
        hit = torch.isinf(out) if value == float("inf") else torch.isnan(out)
        assert bool(hit[1, :, 5].all()) and int(hit.sum()) == 2
    cache = fresh()
    cache.pool[0, 0][page, 0, 7] = float("nan")                      # a key
    out = cache.attend_shared(q, ints(seqs), 0, starts)
    assert bool(torch.isnan(out[:3]).all()) and bool(torch.isfinite(out[3:]).all())
    cache = fresh()                                                  # scores of minus infinity alone in the shared rows
    cache.pool[0, 0][cache.table[0, :18].long(), 0, :, 0] = float("-inf")
    q = torch.ones_like(q)
    out = cache.attend_shared(q, ints(seqs), 0, starts)
    for s in range(3):
        slots = slots_of(cache, s)[288:]
        k, v = (f64(rows_of(cache.pool, slots))[0, j] for j in (0, 1))
        want, mag, dz = H.attend(f64(q[s]), k, v, 0.125)
        assert (np.abs(f64(out[s]) - want) <= half_step(typ) * np.abs(want) + 2.0 ** -15 * mag + tiny(typ)).all()
    cache.pool[0, 0][:, 0, :, 0] = float("-inf")                     # and everywhere: no weights
    assert bool(torch.isnan(cache.attend_shared(q, ints(seqs), 0, starts)).all())


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_shared_infinite_values_of_small_weights(mb, typ):  # noqa: F811
    """Weights from 1 down to 2^-110: an infinite value of any of them in a shared row is infinite in the sum."""
    typ = TYPES[typ]
    for gap in (1.0, 3.0, 5.0, 9.5):                                 # scores 8 k, 11.5 gap powers of two apart
        for sign in (1.0, -1.0):
            cache = grouped(mb, typ, 64, 1, 16, [(96, [4, 9])], 2)
            table = cache.table.long()
            for s in (0, 1):
                cache.pool[0, 0][table[s, :7], 0] = torch.nan_to_num(cache.pool[0, 0][table[s, :7], 0]) * 0.0
            cache.pool[0, 0][table[0, 0], 0, 3] = gap
            cache.pool[0, 1][table[0, 4], 0, 5, 7] = sign * float("inf")
            out = cache.attend_shared(torch.ones(2, 2, 64, dtype=typ, device=DEV), ints([0, 1]), 0, ints([0, 2]))
            assert bool((out[:, :, 7] == sign * float("inf")).all()), (gap, out[:, :, 7])
            out[:, :, 7] = 0.0
            assert bool(torch.isfinite(out).all())


# ----------------------------------------------------------------------------- attention with the sums of its weights

WEIGHS = [
    # type, dh, hk, query heads a key head, page, lens
    ("bf16", 128, 2, 4, 16, [0, 1, 15, 16, 17, 63, 64, 65, 300]),
    ("f16", 64, 1, 1, 16, [5, 0, 1000]),
    ("bf16", 80, 3, 2, 8, [33, 129, 2]),
    ("f16", 96, 2, 8, 24, [200, 31]),
    ("bf16", 192, 1, 3, 64, [1, 700]),
    ("f16", 256, 2, 2, 16, [129, 64, 2000]),
    ("bf16", 128, 1, 16, 5, [77, 13, 0]),
    ("bf16", 64, 1, 40, 1, [50, 3]),
    ("f16", 128, 4, 7, 48, [9000]),
    ("bf16", 64, 2, 17, 1024, [1500, 1023, 1024, 1025]),
    ("f16", 128, 1, 1, 3, [2, 1] * 150),
    ("bf16", 128, 8, 4, 16, [100 + 37 * i for i in range(20)]),
]


def check_weights(weights, before, q, cache, layer, seqs, scale):
    """All of weights: the rows of the sequences in `seqs` have gained what the formula says, the others nothing."""
    want, tol = f64(before).copy(), np.zeros(before.shape)
    for i, s in enumerate(seqs):
        n = int(cache.length[s]) if s >= 0 else 0
        if n:
            k, v = sequence(cache, layer, s)
            _, _, dz = H.attend(f64(q[i]), k, v, scale)
            p = H.attend_weights(f64(q[i]), k, scale)
            want[layer, s, :, :n] += p
            e = 2 * (cache.dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + (n / 16 + 64) * 2.0 ** -23
            tol[layer, s, :, :n] += e * p + 2.0 ** -23 * np.abs(want[layer, s, :, :n]) + 2.0 ** -126 * q.shape[1]
    off = np.abs(f64(weights) - want)
    assert (off <= tol).all(), float((off / np.maximum(tol, 1e-40)).max())


@pytest.mark.parametrize("case", WEIGHS, ids=["-".join(str(v) for v in c[:5]) for c in WEIGHS])
def test_attend_weigh_matches_the_formula(mb, case):  # noqa: F811
    typ, dh, hk, group, page, lens = case
    typ = TYPES[typ]
    cache = filled(mb, typ, dh, hk, page, lens, 5, layers=2)
    seqs = list(range(len(lens) - 1, -1, -1)) + [-1, 0]
    q = randn(gen(6), len(seqs), hk * group, dh, typ=typ) * 1.5
    before = torch.rand(2, len(lens), hk, cache.table.shape[1] * page, generator=gen(7), device=DEV) * 0.1
    weights, out = before.clone(), torch.full_like(q, 3.0)
    cache.attend_weigh(q, ints(seqs), 1, weights, out=out)
    check(out, q, cache, 1, seqs, dh ** -0.5, typ)
    check_weights(weights, before, q, cache, 1, seqs, dh ** -0.5)
    assert torch.equal(out, cache.attend(q, ints(seqs), 1, out=torch.full_like(q, 3.0)))      # the same attention
    again, (qv, _), (ov, base) = before.clone(), place(q, "packed"), place(torch.full_like(q, 7.0), "packed")
    cache.attend_weigh(qv, ints(seqs), 1, again, out=ov)
    assert torch.equal(again, weights)                                                        # repeatable
    ok = [i for i, s in enumerate(seqs) if s >= 0]
    assert torch.equal(ov[ok], out[ok])
    ov.fill_(7.0)
    assert bool((base == 7.0).all())
    cache.check()


def test_attend_weigh_of_a_sequence_in_several_rows_and_of_bad_ones(mb):  # noqa: F811
    cache = filled(mb, torch.bfloat16, 64, 2, 16, [700, 3, 0, 90], 2)
    seqs = [3, 0, 3, -1, 1, 0, 3, 2, 0]
    q = randn(gen(1), len(seqs), 4, 64, typ=torch.bfloat16)
    weights = torch.zeros(1, 4, 2, cache.table.shape[1] * 16, device=DEV)
    weights[:, :, :, 700:] = float("nan")                            # behind every length: neither read nor written
    before = weights.clone()
    cache.attend_weigh(q, ints(seqs), 0, weights)
    cache.check()
    inside = before.clone()
    check_weights(torch.nan_to_num(weights), torch.nan_to_num(inside), q, cache, 0, seqs, 0.125)
    assert bool(torch.isnan(weights[:, :, :, 700:]).all())
    again = before.clone()
    cache.attend_weigh(q, ints([9, 0, -7, -1, 1, 4, -1, 2, -1]), 0, again)
    assert cache.status() == mb.MAP_EINTERNAL
    check_weights(torch.nan_to_num(again), torch.nan_to_num(inside), q, cache, 0, [-1, 0, -1, -1, 1, -1, -1, 2, -1], 0.125)
    cache.length[0] = 1 << 20
    again = before.clone()
    cache.attend_weigh(q[:1], ints([0]), 0, again)
    assert cache.status() == mb.MAP_EINTERNAL and torch.equal(torch.nan_to_num(again), torch.nan_to_num(before))
    for bad in (weights[:, :3], weights.double(), weights[..., :-1], weights[0]):
        with pytest.raises(ValueError):
            cache.attend_weigh(q, ints(seqs), 0, bad)
    assert cache.attend_weigh(q[:0], ints([]), 0, weights).shape == (0, 4, 64)


def test_attend_weigh_values_at_the_edges(mb):  # noqa: F811
    cache = filled(mb, torch.float16, 64, 1, 16, [100, 40], 2)
    q = torch.ones(2, 2, 64, dtype=torch.float16, device=DEV)
    weights = torch.zeros(1, 2, 1, cache.table.shape[1] * 16, device=DEV)
    cache.attend_weigh(q, ints([0, 1]), 0, weights, scale=0.0)       # 2 query heads: 2 / n each, to an ulp or two
    assert bool(((weights[0, 0, 0, :100] * 50 - 1).abs() <= 2.0 ** -21).all()) and bool((weights[0, 0, 0, 100:] == 0).all())
    weights.zero_()
    cache.pool[0, 0][cache.table[0, 3].long(), 0, 5] = 50.0          # one row takes all
    cache.attend_weigh(q, ints([0, 1]), 0, weights)
    assert float(weights[0, 0, 0, 53]) == 2.0 and float(weights[0, 0].sum()) == 2.0
    cache.pool[0, 0][cache.table[0, 3].long(), 0, 5, 0] = float("nan")
    weights.zero_()
    cache.attend_weigh(q, ints([0, 1]), 0, weights)
    assert bool(torch.isnan(weights[0, 0, 0, :100]).all()) and bool(torch.isfinite(weights[0, 1]).all())
    cache.pool[0, 0][cache.table[0, 3].long(), 0, 5, 0] = float("-inf")
    weights.zero_()
    cache.attend_weigh(q, ints([0, 1]), 0, weights)
    assert float(weights[0, 0, 0, 53]) == 0.0 and abs(float(weights[0, 0].sum()) - 2.0) <= 2 * (100 / 16 + 64) * 2.0 ** -23 + 2.0 ** -18


# ----------------------------------------------------------------------------- eviction

def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def run_evict(mb, cache, model, weights, seqs, first, last, k):  # noqa: F811
    """The call against the model: state, pool and weights.  Returns whether it was done."""
    before, after, w = cache.pool.clone(), cache.pool.clone(), weights.cpu().numpy().copy()
    none = first is None
    moves = model.evict(seqs, [0] * len(seqs) if none else first, [0] * len(seqs) if none else last, k, w)
    cache.evict(weights, ints(seqs), None if none else ints(first), None if none else ints(last), k)
    page = cache.page
    for layer, head, to, at in moves or []:
        to, at = (torch.tensor(x, dtype=torch.int64, device=DEV) for x in (to, at))
        for kv in (0, 1):
            after[layer, kv][to // page, head, to % page] = before[layer, kv][at // page, head, at % page]
    same_state(cache, model)
    np.testing.assert_array_equal(weights.cpu().numpy(), w)
    assert same_bits(cache.pool, after)
    return moves is not None


@pytest.mark.parametrize("page,dh,hk,layers,seed", [(16, 128, 2, 2, 0), (1, 8, 1, 1, 1), (5, 40, 3, 2, 2), (64, 64, 8, 1, 3),
                                                    (100, 16, 1, 1, 4), (7, 256, 1, 3, 5), (24, 96, 4, 2, 6)])
def test_evict_follows_the_model(mb, page, dh, hk, layers, seed):  # noqa: F811
    """Runs of extensions, forks, evictions and frees, good and refused ones."""
    import random
    r = random.Random(seed)
    pages, seqs, max_pages = 60, 7, 12
    cache = mb.Cache.empty(layers, pages, hk, page, dh, seqs, max_pages, torch.float16)
    cache.pool.normal_(generator=gen(seed))
    weights = torch.zeros(layers, seqs, hk, max_pages * page, device=DEV)
    model = H.Pages(pages, page, seqs, max_pages)
    done = refused = 0
    for step in range(60):
        who = [s for s in range(seqs) if model.length[s] == 0]
        for s in r.sample(who, min(2, len(who))):
            parents = [p for p in range(seqs) if model.length[p]]
            if parents and r.random() < 0.7:
                p = r.choice(parents)
                if model.fork([p], [s]) is not None:
                    cache.fork(ints([p]), ints([s]))
            n = r.randint(0, 5 * page)
            if model.extend([s], [n], n) is not None:
                cache.extend(ints([s]), ints([n]), rows=n)
            else:
                cache.extend(ints([s]), ints([n]), rows=n)
                assert cache.status() == mb.MAP_ENOMEM
        cache.check()
        same_state(cache, model)
        g = gen(1000 * seed + step)
        cache.pool.normal_(generator=g)
        weights.uniform_(generator=g)
        style = r.random()
        if style < 0.3:
            weights.mul_(4).floor_()                                 # many equal ones
        elif style < 0.5:
            weights.sub_(0.5)
            weights[weights > 0.4] = float("nan")
            weights[weights < -0.45] = float("-inf")
        elif style < 0.6:
            weights.mul_(1e-44)                                      # subnormal
        elif style < 0.7:
            weights.zero_()
            weights[..., ::2] = -0.0
        n = r.randint(0, 5)
        ask = [r.choice(range(seqs)) for _ in range(n)] if r.random() < 0.1 else r.sample(range(seqs), n)
        ask = [-1 if r.random() < 0.1 else s for s in ask]
        if r.random() < 0.04 and ask:
            ask[0] = r.choice([seqs, -2])
        first, last = ([r.choice([0, 0, 1, page, r.randint(0, 2 * page)]) for _ in ask] for _ in range(2))
        if r.random() < 0.05 and ask:
            r.choice([first, last])[0] = -1
        if r.random() < 0.2:
            first = last = None
        k = r.choice([0, 1, 2, page, r.randint(0, 4 * page)])
        ok = run_evict(mb, cache, model, weights, ask, first, last, k)
        assert cache.status() in ((mb.MAP_OK,) if ok else (mb.MAP_ENOMEM, mb.MAP_EINTERNAL))
        done, refused = done + ok, refused + (not ok)
        if r.random() < 0.5:
            gone = [r.randrange(seqs)]
            cache.free(ints(gone))
            model.free(gone)
    assert done > 20 and done + refused == 60


@pytest.mark.parametrize("page,dh,hk,lens,first,last,k", [
    (16, 64, 2, [9000], 3, 100, 2500), (64, 128, 1, [20000, 1, 4097], 0, 0, 4096), (24, 96, 3, [3000, 2999, 50], 35, 7, 100),
    (16, 8, 1, [40001], 4, 4, 39000), (1024, 256, 1, [5000], 1000, 1024, 0), (3, 16, 2, [2049, 1025], 1, 0, 1024)])
def test_evict_of_long_sequences(mb, page, dh, hk, lens, first, last, k):  # noqa: F811
    typ = torch.bfloat16
    cache = filled(mb, typ, dh, hk, page, lens, 3)
    model = H.Pages(cache.refs.shape[0], page, len(lens), cache.table.shape[1])
    model.length, model.refs = list(lens), cache.refs.cpu().tolist()
    model.table = [cache.table[s, : -(-t // page)].cpu().tolist() for s, t in enumerate(lens)]
    weights = torch.exp(2.5 * torch.randn(1, len(lens), hk, cache.table.shape[1] * page, generator=gen(1), device=DEV))
    weights[:, :, 0] = (weights[:, :, 0] * 4).floor()                # thousands of equal ones
    n = len(lens)
    assert run_evict(mb, cache, model, weights, list(range(n)), [first] * n, [last] * n, k)
    cache.check()


def test_evict_refuses_what_it_cannot_do_whole(mb):  # noqa: F811
    def fresh():
        c = grouped(mb, torch.float16, 64, 1, 16, [(64, [5, 40]), (0, [100])], 1, spare=-2)       # (four pages are held twice: two are free)
        return c, torch.rand(1, 3, 1, c.table.shape[1] * 16, generator=gen(1), device=DEV)

    def nothing_changes(code, *args):
        state = [t.clone() for t in (cache.pool.view(torch.int16), cache.length, cache.refs, weights)]
        cache.evict(weights, *args)
        assert cache.status() == code
        assert all(torch.equal(a, b) for a, b in zip(state, (cache.pool.view(torch.int16), cache.length, cache.refs, weights)))

    cache, weights = fresh()
    nothing_changes(mb.MAP_ENOMEM, ints([0, 2]), None, None, 40)     # three shared pages to replace, two free
    nothing_changes(mb.MAP_EINTERNAL, ints([2, 2]), None, None, 4)
    nothing_changes(mb.MAP_EINTERNAL, ints([2, 3]), None, None, 4)
    nothing_changes(mb.MAP_EINTERNAL, ints([2, -2]), None, None, 4)
    nothing_changes(mb.MAP_EINTERNAL, ints([2]), ints([-1]), ints([0]), 4)
    nothing_changes(mb.MAP_EINTERNAL, ints([2]), ints([0]), ints([-1]), 4)
    nothing_changes(mb.MAP_OK, ints([-1]), None, None, 4)
    nothing_changes(mb.MAP_OK, ints([0, 1, 2]), None, None, 104)     # as many as there are
    nothing_changes(mb.MAP_OK, ints([0, 1, 2]), ints([200] * 3), ints([1 << 30] * 3), 0)
    nothing_changes(mb.MAP_OK, ints([0, 1, 2]), ints([(1 << 31) - 1] * 3), ints([(1 << 31) - 1] * 3), 0)
    for bad in (-1, 1 << 20):
        cache.length[2] = bad
        nothing_changes(mb.MAP_EINTERNAL, ints([1, 2]), ints([64, 0]), ints([0, 0]), 4)
    cache.length[2] = 100
    for bad in (-1, cache.pool.shape[2], 1 << 30):
        cache.table[2, 5] = bad
        nothing_changes(mb.MAP_EINTERNAL, ints([1, 2]), ints([64, 0]), ints([0, 0]), 4)
    cache, weights = fresh()
    for bad in (weights[:, :2], weights.double(), weights[..., 1:]):
        with pytest.raises(ValueError):
            cache.evict(bad, ints([0]), None, None, 1)
    with pytest.raises(ValueError):
        cache.evict(weights, ints([0]), ints([0, 0]), None, 1)
    with pytest.raises(mb.MapError):
        cache.evict(weights, ints([0]), None, None, -1)
    cache.evict(weights, ints([]), None, None, 1)
    cache.evict(weights, ints([0, 2]), ints([64, 0]), ints([0, 0]), 1)       # behind the shared pages: in place
    cache.check()
    assert cache.length.cpu().tolist() == [65, 104, 1]


def test_evict_of_many_sequences(mb):  # noqa: F811
    """More entries than a block has threads, every third the fork of another, some padding, some left as they are."""
    n, page, hk = 2100, 4, 2
    cache = mb.Cache.empty(1, 40000, hk, page, 16, n, 16)
    cache.pool.normal_(generator=gen(1))
    model = H.Pages(40000, page, n, 16)
    own = [s for s in range(n) if s % 3]
    lens = [(7 * s) % 53 for s in own]
    cache.extend(ints(own), ints(lens), rows=sum(lens))
    model.extend(own, lens, sum(lens))
    forks = [s for s in range(n) if s % 3 == 0]
    cache.fork(ints([s + 1 for s in forks]), ints(forks))
    for to, at in model.fork([s + 1 for s in forks], forks):
        assert to >= 0 and at >= 0
    weights = torch.rand(1, n, hk, 16 * page, generator=gen(2), device=DEV)
    ask = [-1 if s % 11 == 0 else s for s in range(n - 1, -1, -1)]
    first, last = [s % 3 for s in range(n)], [s % 5 for s in range(n)]
    assert run_evict(mb, cache, model, weights, ask, first, last, 9)
    cache.check()


def test_evict_past_32_bits(mb):  # noqa: F811
    """The last pages of a pool of 2^33 bytes."""
    dh, hk, page = 128, 8, 64
    pages = (1 << 32) // (4 * hk * page * dh) + 3
    cache = mb.Cache.empty(2, pages, hk, page, dh, 3, 4)
    cache.refs[: pages - 3] = 1
    cache.extend(ints([0]), ints([150]), rows=150)
    slots = slots_of(cache, 0)
    assert min(slots) // page == pages - 3
    where = torch.tensor(slots, device=DEV)
    rows = randn(gen(1), 2, 2, hk, 150, dh, typ=torch.bfloat16)
    for l in range(2):
        for kv in range(2):
            cache.pool[l, kv][where // page, :, where % page] = rows[l, kv].transpose(0, 1)
    weights = torch.rand(2, 3, hk, 256, generator=gen(2), device=DEV)
    order = weights[:, 0, :, 10:140].argsort(dim=-1, descending=True)[..., :50].sort(dim=-1).values + 10
    cache.evict(weights, ints([0]), ints([10]), ints([10]), 50)
    cache.check()
    got = rows_of(cache.pool, slots_of(cache, 0))                    # [layers, 2, rows, heads, dh]
    head = torch.arange(10, device=DEV).expand(2, hk, -1)
    src = torch.cat((head, order, head + 140), -1)
    want = rows.gather(3, src[:, None, :, :, None].expand(2, 2, -1, -1, dh)).transpose(2, 3)
    assert torch.equal(got, want)


# ----------------------------------------------------------------------------- together, streams, graphs

def decode(cache, plan, weights, seqs, starts, first, last, steps, q, k, v, outs):
    """Steps of decoding: rows appended, two layers attended (one shared, one weighed); a window cut to 20 rows at the end."""
    for step in range(steps):
        slots = cache.extend(seqs)
        pos = cache.length[None, : seqs.shape[0]].contiguous()
        q0 = plan.append(q[step, 0], k[step, 0], v[step, 0], pos, cache, 0, slots)
        q1 = plan.append(q[step, 1], k[step, 1], v[step, 1], pos, cache, 1, slots)
        cache.attend_shared(q0, seqs, 0, starts, out=outs[step, 0])
        cache.attend_weigh(q1, seqs, 1, weights, out=outs[step, 1])
    cache.evict(weights, seqs, first, last, 20)


def test_questions_decode_over_one_image_within_a_budget(mb):  # noqa: F811
    """Forks of one cached image decode together, their caches are cut and they decode on: eager, from the definition, and captured
    and replayed with other rows."""
    dh, hk, hq, page, image, steps, n = 64, 2, 8, 16, 330, 3, 4
    seqs, starts = ints([0, 1, 2, -1]), ints([0, 4])
    first, last = ints([5] * n), ints([3] * n)
    plan = mb.Rope(dh, [0.9 ** i for i in range(32)])
    caches, weights = [], []
    for _ in range(2):
        c = mb.Cache.empty(2, 120, hk, page, dh, 6, 24, torch.float16)
        c.pool.normal_(generator=gen(3))
        c.extend(ints([5]), ints([image]), rows=image)
        c.fork(ints([5] * 3), ints([0, 1, 2]))
        caches.append(c)
        weights.append(torch.zeros(2, 6, hk, 24 * page, device=DEV))
    shape = (steps, 2, n)
    q, k, v = (torch.zeros(*shape, h, dh, dtype=torch.float16, device=DEV) for h in (hq, hk, hk))
    outs = [torch.full((*shape, hq, dh), 3.0, dtype=torch.float16, device=DEV) for _ in range(2)]

    def feed(i):
        for x, t in enumerate((q, k, v)):
            t.copy_(randn(gen(10 * i + x), *t.shape, typ=torch.float16))

    # one pass by hand against the definition
    feed(0)
    c, w = mb.Cache.empty(2, 120, hk, page, dh, 6, 24, torch.float16), weights[0].clone()
    c.pool.copy_(caches[0].pool)
    c.extend(ints([5]), ints([image]), rows=image)
    c.fork(ints([5] * 3), ints([0, 1, 2]))
    for step in range(steps):
        slots = c.extend(seqs)
        pos = c.length[None, :n].contiguous()
        rot = [plan.append(q[step, l], k[step, l], v[step, l], pos, c, l, slots) for l in (0, 1)]
        check(c.attend_shared(rot[0], seqs, 0, starts), rot[0], c, 0, [0, 1, 2, -1], dh ** -0.5, torch.float16)
        before = w.clone()
        check(c.attend_weigh(rot[1], seqs, 1, w), rot[1], c, 1, [0, 1, 2, -1], dh ** -0.5, torch.float16)
        check_weights(w, before, rot[1], c, 1, [0, 1, 2, -1], dh ** -0.5)
    kept = w[1, 0, 0, 5: image + steps - 3].argsort(descending=True, stable=True)[:20].sort().values + 5
    keys = rows_of(c.pool, slots_of(c, 0))[1, 0, :, 0]
    c.evict(w, seqs, first, last, 20)
    c.check()
    assert c.length.cpu().tolist() == [28, 28, 28, 0, 0, image]
    assert torch.equal(rows_of(c.pool, slots_of(c, 0))[1, 0, 5:25, 0], keys[kept])
    image_rows = rows_of(c.pool, slots_of(c, 5))
    assert torch.equal(image_rows, rows_of(caches[0].pool, slots_of(caches[0], 5)))          # the image stays whole
    # the same eager and captured
    args = (plan, weights[0], seqs, starts, first, last, steps, q, k, v)
    eager, want = caches[0], []
    for i in range(3):
        feed(i)
        outs[0].fill_(3.0)
        decode(eager, *args, outs[0])
        want.append(outs[0].clone())
    eager.check()
    torch.cuda.synchronize()
    g, warm = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=warm):
        decode(caches[1], plan, weights[1], *args[2:], outs[1])
    for i in range(3):
        feed(i)
        outs[1].fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[1], want[i]), i
    caches[1].check()
    assert torch.equal(caches[1].length, eager.length) and torch.equal(caches[1].refs, eager.refs)
    assert torch.equal(weights[1], weights[0])


def test_decode_calls_on_a_stream_of_the_callers(mb):  # noqa: F811
    groups = [(500, [9, 40, 3]), (64, [1, 1])]
    cache = grouped(mb, torch.bfloat16, 128, 2, 16, groups, 2)
    seqs, starts, st = ints(range(5)), ints(starts_of(groups)), torch.cuda.Stream()
    q = randn(gen(1), 5, 8, 128, typ=torch.bfloat16)
    weights = [torch.rand(1, 5, 2, cache.table.shape[1] * 16, generator=gen(2), device=DEV)]
    weights.append(weights[0].clone())
    want = cache.attend_shared(q, seqs, 0, starts), cache.attend_weigh(q, seqs, 0, weights[0])
    torch.cuda.synchronize()
    for _ in range(20):
        busy = torch.zeros(1 << 26, device=DEV)
        st.wait_stream(torch.cuda.current_stream())
        w = weights[1].clone()
        st.wait_stream(torch.cuda.current_stream())
        got = cache.attend_shared(q.clone(), seqs.clone(), 0, starts.clone(), stream=st), cache.attend_weigh(q.clone(), seqs, 0, w, stream=st)
        junk = [torch.full_like(q, 9.0) for _ in range(8)]           # where dropped inputs or workspaces would lie
        torch.cuda.current_stream().wait_stream(st)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(w, weights[0])
        del busy, junk
    cache.evict(weights[1], seqs[:1], None, None, 40, stream=st)
    st.synchronize()
    cache.check(stream=st)
    assert int(cache.length[0]) == 40


def test_workspaces_that_grow_between_a_graphs_replays(mb):  # noqa: F811
    """A graph's calls have memory of their own: eager calls before, between and after its replays may need more and less."""
    groups = [(500, [9, 40, 3]), (64, [1, 1])]
    cache = grouped(mb, torch.bfloat16, 128, 2, 16, groups, 2, spare=200, room=10)
    few, many = ints([0, 1]), ints(list(range(5)) * 40)
    q = [randn(gen(i), n, 8, 128, typ=torch.bfloat16) for i, n in enumerate((2, 200))]
    starts = [ints([0, 2]), ints([0, 200])]
    weights = torch.zeros(1, 5, 2, cache.table.shape[1] * 16, device=DEV)
    want = [cache.attend_shared(q[0], few, 0, starts[0]), cache.attend(q[1], many, 0)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = cache.attend_shared(q[0], few, 0, starts[0]), cache.attend_weigh(q[0], few, 0, weights)
    for _ in range(3):
        g.replay()
        a, b = cache.attend_weigh(q[1], many, 0, weights), cache.attend_shared(q[1], many, 0, starts[1])
        g.replay()
        c = cache.attend_shared(q[0], few, 0, starts[0])
        torch.cuda.synchronize()
        assert torch.equal(a, want[1]) and torch.equal(c, want[0]) and torch.equal(held[0], want[0])
        check(b, q[1], cache, 0, many.tolist(), 128 ** -0.5, torch.bfloat16)
    cache.evict(weights, many[:5], None, None, 30)
    g.replay()
    check(held[0], q[0], cache, 0, [0, 1], 128 ** -0.5, torch.bfloat16)
    cache.check()
    assert cache._kept.shape[0] <= 1 << 26


@pytest.mark.parametrize("call", ["shared", "weigh", "evict"])
def test_decode_calls_of_two_caches_from_two_threads(mb, call):  # noqa: F811
    calls, held = [], []
    for dh, group in ((64, 16), (256, 1)) * 2:
        c, st = grouped(mb, torch.float16, dh, 1, 16, [(200, [40, 20])], 3), torch.cuda.Stream()
        seqs, starts = ints([0, 1]), ints([0, 2])
        q = randn(gen(4), 2, group, dh, typ=torch.float16)
        out = torch.empty_like(q)
        w = torch.zeros(1, 2, 1, c.table.shape[1] * 16, device=DEV)
        heads, oheads = (mb._heads(t, 2, dh, q.dtype, q.device) for t in (q, out))
        lib, ws_of = mb.lib, lambda size: torch.empty(size, dtype=torch.uint8, device=DEV)
        if call == "shared":
            ws = ws_of(lib.map_cache_attend_shared_workspace(c.desc, group, 2, 1))
            args = (c.desc, 0, heads, seqs.data_ptr(), 2, starts.data_ptr(), 1, dh ** -0.5, oheads, ws.data_ptr(), st.cuda_stream)
            held.append((out, c.attend_shared(q, seqs, 0, starts), ws))
            fn = lib.map_cache_attend_shared
        elif call == "weigh":
            ws = ws_of(lib.map_cache_attend_weigh_workspace(c.desc, group, 2))
            args = (c.desc, 0, heads, seqs.data_ptr(), 2, dh ** -0.5, oheads, w.data_ptr(), ws.data_ptr(), st.cuda_stream)
            held.append((out, c.attend(q, seqs, 0), ws))
            fn = lib.map_cache_attend_weigh
        else:
            ws = ws_of(lib.map_cache_evict_workspace(c.desc, 2, 1000))
            args = (c.desc, w.data_ptr(), seqs.data_ptr(), 2, None, None, 1000, ws.data_ptr(), st.cuda_stream)
            out.fill_(1.0)
            held.append((out, out.clone(), ws))
            fn = lib.map_cache_evict
        calls.append(lambda fn=fn, args=args, keep=(c, q, seqs, starts, w): fn(*args))
    torch.cuda.synchronize()
    assert together(calls, 5000) == []
    assert all(torch.equal(out, want) for out, want, _ in held)
