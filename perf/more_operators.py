"""What is measured of decoding over a shared and a bounded cache: the operators that answer many questions on one
cached image and keep a long answer's cache within a budget.

  shared   attention of single tokens for groups of sequences that begin with the same pages, whose rows are read once
           for all of a group (`Cache.attend_shared`)
  weigh    attention of single tokens that also adds each row's attention weight to its running sum
           (`Cache.attend_weigh`)
  evict    the rows with the least weight leave the cache, layer by layer and head by head (`Cache.evict`)

A case is a dict of plain values.  Sizes are those of this repository's configurations (LLaVA-NeXT: 2880 visual tokens
after 35 of a prompt, 32 heads of 128; LLaVA-1.5: 576; Qwen2.5-VL: up to 1280 tokens, 28 heads of 128), of language models'
usual head layouts, and odd ones.  Lengths that differ between the sequences of a batch are the case's own, so that output
shapes are; values come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
SIZE = 2                                   # bytes of an element of either type


# ----------------------------------------------------------------------------- cases

def listed() -> list:
    return [
        # Four questions on one LLaVA-1.5 image, decoding together: the smallest call.
        dict(name="shared_4q_n576", op="shared", groups=1, each=4, p_lo=611, p_hi=611, t_lo=9, t_hi=60, hq=32, hk=32,
             dh=128, page=16, type="bf16"),
        # Sixty-four questions on one LLaVA-NeXT image that stays whole.
        dict(name="shared_64q_n2880", op="shared", groups=1, each=64, p_lo=2915, p_hi=2915, t_lo=20, t_hi=300, hq=32,
             hk=8, dh=128, page=16, type="bf16"),
        # Images of different sizes with eight questions each.
        dict(name="shared_8x8_n1280", op="shared", groups=8, each=8, p_lo=290, p_hi=1315, t_lo=1, t_hi=400, hq=28, hk=4,
             dh=128, page=32, type="bf16"),
        # Thirty-two samples of answers on one long video.
        dict(name="shared_32_long", op="shared", groups=1, each=32, p_lo=60001, p_hi=60001, t_lo=100, t_hi=700, hq=28,
             hk=4, dh=128, page=64, type="f16"),
        # One short dialogue: latency.
        dict(name="weigh_one_n700", op="weigh", seqs=1, t_lo=701, t_hi=701, hq=28, hk=4, dh=128, page=16, type="bf16"),
        # Sixty-four pruned prompts with answers of different lengths.
        dict(name="weigh_b64", op="weigh", seqs=64, t_lo=200, t_hi=1600, hq=32, hk=8, dh=128, page=16, type="bf16"),
        # Heads of 96 columns over pages that are no power of two, odd lengths.
        dict(name="weigh_b7_odd", op="weigh", seqs=7, t_lo=1, t_hi=5001, hq=40, hk=10, dh=96, page=24, type="f16"),
        # One long video dialogue: the split over one sequence.
        dict(name="weigh_one_long", op="weigh", seqs=1, t_lo=120001, t_hi=120001, hq=28, hk=4, dh=128, page=64,
             type="f16"),
        # One answer's cache back to its budget, all 28 layers: the smallest eviction.
        dict(name="evict_one_n1100", op="evict", seqs=1, t_lo=1100, t_hi=1100, first=4, last=128, k=380, layers=28, hk=4,
             dh=128, page=16, shared=False, type="bf16"),
        # A batch of long answers, each cut to a little more than a quarter.
        dict(name="evict_b6_n4096", op="evict", seqs=6, t_lo=3001, t_hi=4096, first=35, last=256, k=1024, layers=28,
             hk=4, dh=128, page=16, shared=False, type="bf16"),
        # Eight questions forked from one cached LLaVA-NeXT image: each takes pages of its own for what it keeps.
        dict(name="evict_8q_n2880", op="evict", seqs=8, t_lo=2915, t_hi=3000, first=35, last=50, k=160, layers=32, hk=8,
             dh=128, page=16, shared=True, type="bf16"),
        # One long video dialogue in eight layers.
        dict(name="evict_one_long", op="evict", seqs=1, t_lo=60001, t_hi=60001, first=4, last=512, k=16384, layers=8,
             hk=4, dh=128, page=64, shared=False, type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng) -> dict:
    op = rng.choice(["shared", "weigh", "evict"])
    typ = rng.choice(["bf16", "bf16", "f16"])
    hk = rng.choice([1, 2, 4, 8, 10])
    dh = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    page = rng.choice([8, 16, 16, 24, 32, 64, 100])
    if op == "evict":
        t_hi = _log(rng, 16, 60000)
        t_lo = max(1, t_hi // rng.choice([1, 2, 10]))
        first, last = rng.choice([0, 4, 35]), _log(rng, 1, max(2, t_hi // 3)) - 1
        return dict(op=op, seqs=_log(rng, 1, 16), t_lo=t_lo, t_hi=t_hi, first=first, last=last,
                    k=_log(rng, 1, max(2, t_hi // 2)) - 1, layers=rng.choice([1, 4, 8, 28]), hk=hk, dh=dh, page=page,
                    shared=rng.random() < 0.4, type=typ)
    hq = hk * rng.choice([1, 2, 4, 7, 8])
    if op == "weigh":
        t_hi = _log(rng, 4, 60000)
        return dict(op=op, seqs=_log(rng, 1, max(1, min(128, 200000 // t_hi))), t_lo=max(1, t_hi // rng.choice([1, 4, 50])),
                    t_hi=t_hi, hq=hq, hk=hk, dh=dh, page=page, type=typ)
    each = _log(rng, 2, 64)
    p_hi = _log(rng, 16, max(17, min(60000, 400000 // each)))
    t_hi = _log(rng, 1, 1000)
    return dict(op=op, groups=_log(rng, 1, max(1, min(16, 400000 // (each * (p_hi + t_hi))))), each=each,
                p_lo=max(1, p_hi // rng.choice([1, 4])), p_hi=p_hi, t_lo=max(1, t_hi // rng.choice([1, 4])), t_hi=t_hi, hq=hq,
                hk=hk, dh=dh, page=page, type=typ)


def draw(rng) -> dict:
    """One more case: sizes spread over the ranges, no costlier than the largest listed one of its operator."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = tuple(map(max, most.get(c["op"], (0, 0)), (w["bytes"], w["flops"])))
    while True:
        c = _drawn(rng)
        w = work(c)
        if 0 < w["bytes"] <= most[c["op"]][0] and w["flops"] <= most[c["op"]][1] and _bytes_held(c) <= 4e9:
            return c


# ----------------------------------------------------------------------------- sizes that a case fixes

def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case):
    """Rows of each sequence and, for shared, of each group's common beginning."""
    r = _rng(case)
    if case["op"] != "shared":
        return [r.randint(case["t_lo"], case["t_hi"]) for _ in range(case["seqs"])], []
    prefix = [r.randint(case["p_lo"], case["p_hi"]) for _ in range(case["groups"])]
    return [p + r.randint(case["t_lo"], case["t_hi"]) for p in prefix for _ in range(case["each"])], prefix


def _evicted(case, t):
    """Rows of a sequence of t rows before which none moves, rows that may leave, and its rows afterwards."""
    window = max(0, t - case["first"] - case["last"])
    return case["first"], window, t - window + min(window, case["k"])


def _row_bytes(case):
    return 2 * case["hk"] * case["dh"] * SIZE


def _bytes_held(case):
    """What the plain form holds at its largest, roughly."""
    lens, _ = _lens(case)
    if case["op"] == "evict":
        return 3 * case["layers"] * _row_bytes(case) * sum(lens)
    return 3 * _row_bytes(case) * len(lens) * max(lens) + 12 * case["hq"] * len(lens) * max(lens)


def work(case) -> dict:
    lens, prefix = _lens(case)
    if case["op"] == "evict":
        units, moved, weights = case["layers"] * case["hk"], 0, 0
        for t in lens:
            first, window, left = _evicted(case, t)
            if left < t:
                moved += left - first
                weights += window + t - first                   # read once; written where rows were
        return {"bytes": units * (moved * 2 * 2 * case["dh"] * SIZE + weights * 4), "flops": 0}
    distinct = sum(lens)
    for i, p in enumerate(prefix):                              # whole pages of a group's beginning are held once
        distinct -= (case["each"] - 1) * (p // case["page"] * case["page"])
    bytes_ = distinct * _row_bytes(case) + 2 * len(lens) * case["hq"] * case["dh"] * SIZE
    if case["op"] == "weigh":
        bytes_ += 8 * sum(lens) * case["hk"]
    return {"bytes": bytes_, "flops": 4 * sum(lens) * case["hq"] * case["dh"]}


# ----------------------------------------------------------------------------- inputs

def _gen(seed: int) -> torch.Generator:
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 29) % (1 << 62))


def _sum_of_weights(g, *shape):
    """Running sums of attention weights: over many orders of magnitude, and some rows that no token has looked at."""
    w = torch.exp(2.5 * torch.randn(*shape, generator=g, device=DEV)) / 256
    return torch.where(torch.rand(*shape, generator=g, device=DEV) < 0.03, torch.zeros_like(w), w)


def prepare(case, seed) -> dict:
    g = _gen(seed)
    s = {"case": dict(case)}
    lens, prefix = _lens(case)
    n, page, hk, dh = len(lens), case["page"], case["hk"], case["dh"]
    # which sequences share their first pages, and how many
    each = case["each"] if case["op"] == "shared" else n if case.get("shared") else 1
    if case["op"] == "shared":
        shared = [p // page for p in prefix]
    else:
        shared = [min(lens) // page if case.get("shared") else 0] * (n // each)
    used = [-(-t // page) for t in lens]
    need = sum(shared) + sum(u - shared[i // each] for i, u in enumerate(used))
    spare = n * (-(-max(_evicted(case, t)[2] for t in lens) // page) + 1) if case.get("shared") else 3
    pages, max_pages = need + spare, max(used) + 1
    layers = case.get("layers", 1)
    typ = TYPES[case["type"]]
    s["pool"] = torch.empty(layers, 2, pages, hk, page, dh, dtype=typ, device=DEV)
    for plane in s["pool"].flatten(0, 1):
        plane.normal_(generator=g)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    # the page table, lengths and holders of each page: views of one array
    s["book"] = torch.zeros(n * max_pages + n + pages, dtype=torch.int32, device=DEV)
    s["table"] = s["book"][: n * max_pages].view(n, max_pages)
    s["length"] = s["book"][n * max_pages: n * max_pages + n]
    s["refs"] = s["book"][n * max_pages + n:]
    at = 0
    for i, u in enumerate(used):
        k = shared[i // each]
        if i % each == 0:
            first, at = order[at: at + k], at + k
            s["refs"][first.long()] = each
        s["table"][i, :k] = first
        s["table"][i, k: u] = order[at: at + u - k]
        s["refs"][order[at: at + u - k].long()] = 1
        at += u - k
    s["length"].copy_(torch.tensor(lens, dtype=torch.int32))
    s["lens"] = lens
    s["seqs"] = torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    if case["op"] != "shared":
        w = _sum_of_weights(g, layers, n, hk, max_pages * page)
        behind = torch.arange(max_pages * page, device=DEV)[None] >= s["length"][:, None]
        s["weights"] = w.masked_fill_(behind[None, :, None], 0.0)
    if case["op"] == "evict":
        # a pass changes these: the next one finds the sequences as long as they were, with other sums
        s["book_before"], s["weights_before"] = s["book"].clone(), s["weights"].clone()
        s["first"], s["last"] = (torch.full((n,), case[x], dtype=torch.int32, device=DEV) for x in ("first", "last"))
    else:
        s["q"] = torch.randn(n, case["hq"], dh, generator=g, device=DEV, dtype=typ) * 2
    if case["op"] == "shared":
        s["starts"] = torch.arange(0, n + 1, each, dtype=torch.int32, device=DEV)
    if own:
        from paper_2608_06411_gb300 import binding as mb
        s["cache"] = mb.Cache(s["pool"], s["table"], s["length"], s["refs"])
    return s


# ----------------------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "evict":                      # the rows, and their weights, that have come since the last eviction
        s["book"].copy_(s["book_before"])
        s["weights"].copy_(s["weights_before"])
    if not own:
        return PLAIN[op](s)
    c = s["cache"]
    if op == "shared":
        return c.attend_shared(s["q"], s["seqs"], 0, s["starts"])
    if op == "weigh":
        return c.attend_weigh(s["q"], s["seqs"], 0, s["weights"]), s["weights"]
    c.evict(s["weights"], s["seqs"], s["first"], s["last"], s["case"]["k"])
    return s["pool"], s["table"], s["length"], s["refs"], s["weights"]


# The plain forms: elementary torch operations in fp32, one rounding at the end.

def _softmax(s):
    """Weights [n, hk, group, tokens] of q's rows, and the sequences' values [n, tokens, hk, dh]."""
    q, seqs = s["q"].float(), s["seqs"].long()
    n, hq, dh = q.shape
    pages = s["table"][seqs].long()
    k, v = (s["pool"][0, i][pages].transpose(2, 3).flatten(1, 2).float() for i in (0, 1))
    on = torch.arange(k.shape[1], device=DEV)[None] < s["length"][seqs][:, None]
    z = torch.einsum("nhgd,nthd->nhgt", q.view(n, k.shape[2], -1, dh), k) / math.sqrt(dh)
    z = torch.where(on[:, None, None], z, torch.full_like(z, -math.inf))
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True), torch.where(on[:, :, None, None], v, torch.zeros_like(v))


def _plain_shared(s):
    p, v = _softmax(s)
    return torch.einsum("nhgt,nthd->nhgd", p, v).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_weigh(s):
    p, v = _softmax(s)
    s["weights"][0].index_add_(0, s["seqs"].long(), p.sum(2))
    return torch.einsum("nhgt,nthd->nhgd", p, v).reshape(s["q"].shape).to(s["q"].dtype), s["weights"]


def _plain_evict(s):
    c, page = s["case"], s["case"]["page"]
    layers, _, pages, hk, _, dh = s["pool"].shape
    table, refs, weights = s["table"], s["refs"], s["weights"]
    rows = s["pool"].view(-1, dh)
    layer = torch.arange(layers, device=DEV)[:, None, None]
    head = torch.arange(hk, device=DEV)[None, :, None]
    free = torch.argsort((refs > 0).to(torch.uint8), stable=True)       # page numbers, the free ones first
    holders = refs.clone()
    taken = torch.zeros((), dtype=torch.int64, device=DEV)
    for i, b in enumerate(range(len(s["lens"]) - 1, -1, -1)):           # (the order of seqs)
        t = s["lens"][b]
        first, window, left = _evicted(c, t)
        if left == t:
            continue
        was = table[b].long()
        w = weights[:, b, :, first: first + window]
        kept = w.sort(dim=-1, descending=True, stable=True).indices[..., : c["k"]].sort(dim=-1).values + first
        tail = torch.arange(first + window, t, device=DEV).expand(layers, hk, -1)
        src = torch.cat((torch.arange(first, device=DEV).expand(layers, hk, -1), kept, tail), -1)
        # pages that others hold too are replaced by free ones, the lowest first
        lo, hi, had = first // page, -(-left // page), -(-t // page)
        both = holders[was[lo:hi]] > 1
        rank = both.cumsum(0) - 1 + taken
        now = was.clone()
        now[lo:hi] = torch.where(both, free[rank.clamp(0, free.numel() - 1)], was[lo:hi])
        taken = taken + both.sum()
        table[b] = now.to(torch.int32)
        refs.index_add_(0, was[lo:hi], -both.to(torch.int32))
        refs.index_add_(0, now[lo:hi], both.to(torch.int32))
        refs.index_add_(0, was[hi:had], torch.full((had - hi,), -1, dtype=torch.int32, device=DEV))
        to = torch.arange(left, device=DEV)
        for kv in (0, 1):
            plane = (layer * 2 + kv) * pages
            at = ((plane + was[src // page]) * hk + head) * page + src % page
            put = ((plane + now[to // page]) * hk + head) * page + to % page
            lo_row = lo * page
            rows[put[..., lo_row:]] = rows[at[..., lo_row:]]
        weights[:, b, :, :left] = weights[:, b].gather(-1, src)
        weights[:, b, :, left:t] = 0.0
        s["length"][b] = left
    return s["pool"], table, s["length"], refs, weights


PLAIN = {"shared": _plain_shared, "weigh": _plain_weigh, "evict": _plain_evict}


# ----------------------------------------------------------------------------- 64-bit values

def exact(case, seed):
    s = prepare(case, seed)
    page, pool = case["page"], s["pool"]
    table, lens, refs = s["table"].cpu().numpy(), list(s["lens"]), s["refs"].cpu().numpy()
    if case["op"] != "evict":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        group = case["hq"] // case["hk"]
        sums = s["weights"].double() if case["op"] == "weigh" else None
        for i, b in enumerate(s["seqs"].tolist()):
            at = torch.from_numpy(table[b, : -(-lens[b] // page)].astype("int64")).to(DEV)
            k, v = (pool[0, j][at].double().permute(1, 0, 2, 3).flatten(1, 2)[:, : lens[b]] for j in (0, 1))
            for h in range(case["hk"]):
                mine = slice(h * group, (h + 1) * group)
                p = torch.softmax(s["q"][i, mine].double() @ k[h].T * case["dh"] ** -0.5, -1)
                out[i, mine] = p @ v[h]
                if sums is not None:
                    sums[0, b, h, : lens[b]] += p.sum(0)
        return out if sums is None else (out, sums)
    before, table_was, holders = pool.clone(), table.copy(), refs.copy()
    free = [p for p in range(len(refs)) if refs[p] == 0]
    for b in s["seqs"].tolist():
        t = lens[b]
        window = range(case["first"], t - case["last"])
        if len(window) <= case["k"]:
            continue
        left = t - len(window) + case["k"]
        for j in range(case["first"] // page, -(-t // page)):
            p = table_was[b, j]
            if j * page >= left:
                refs[p] -= 1
            elif holders[p] > 1:
                refs[p] -= 1
                table[b, j] = free.pop(0)
                refs[table[b, j]] = 1
        old, new = (torch.from_numpy(x[b].astype("int64")).to(DEV) for x in (table_was, table))
        to = torch.arange(case["first"] // page * page, left, device=DEV)
        for l in range(case["layers"]):
            for h in range(case["hk"]):
                w = s["weights"][l, b, h]
                # greatest first, of equals the one in front: a row's place is how many come before it
                order = torch.argsort(-w[window.start: window.stop].double(), stable=True)[: case["k"]]
                kept = torch.zeros(len(window), dtype=torch.bool, device=DEV)
                kept[order] = True
                src = torch.cat((torch.arange(window.start, device=DEV), kept.nonzero()[:, 0] + window.start,
                                 torch.arange(window.stop, t, device=DEV)))
                rest = w[src]
                w[:t] = 0.0
                w[:left] = rest
                src = src[to[0]:]
                for kv in (0, 1):
                    pool[l, kv][new[to // page], h, to % page] = before[l, kv][old[src // page], h, src % page]
        s["length"][b] = left
    return pool, torch.from_numpy(table), s["length"], torch.from_numpy(refs), s["weights"]
