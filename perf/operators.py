"""What is measured of the language-model hand-off: the operators that carry a pruned image from `map_select` to a
decoding language model.

  positions    the hand-off sequence with time/height/width position ids (`Context.assemble_axes`)
  rotate       per-head RMS norm of queries and keys with the rotation on several axes (`Rope.rotate`)
  rotate_grad  its gradient (`Rope.grad`)
  append       rotated keys, and values, into a cache's pages (`Cache.extend`, `Rope.append`, `Cache.free`)
  fork         sequences forked from a parent's pages, whole or with the kept tokens of a question, and freed again
               (`Cache.fork`, `Cache.free`)
  attend       attention of single tokens over the pages (`Cache.attend`)

A case is a dict of plain values.  Sizes are those of this repository's configurations (LLaVA-NeXT: 2880 visual tokens,
160 kept, width 4096 = 32 heads of 128; Qwen2.5-VL: up to 1280 tokens, width 3584 = 28 heads of 128), of language
models' usual head layouts, and odd ones.  Lengths that differ between the sequences of a batch are the case's own,
so that output shapes are; values come from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ----------------------------------------------------------------------------- cases

def listed() -> list:
    return [
        # One LLaVA-1.5 image handed to a language model with three position axes: the smallest call.
        dict(name="positions_b1_n576", op="positions", images=1, frames=1, side_lo=24, side_hi=24, D=4096, k=32,
             m_lo=32, m_hi=32),
        # A batch of 16 variable-resolution images (the repository's ragged configuration), 128 kept tokens each.
        dict(name="positions_b16_n1024", op="positions", images=16, frames=1, side_lo=20, side_hi=32, D=3584, k=128,
             m_lo=16, m_hi=128),
        # One decoding step's rows of 8 sequences with grouped heads: latency.
        dict(name="rotate_8rows", op="rotate", rows=8, hq=28, hk=4, dh=128, rot=128, axes=3, mixed=False, adjacent=False,
             norm=True, packed=True, far=4096, type="bf16"),
        # The prompts of 64 pruned LLaVA-NeXT images (160 kept + about 136 question tokens), as many keys as queries,
        # queries and keys in one projection's output.
        dict(name="rotate_b64_prompt", op="rotate", rows=18944, hq=32, hk=32, dh=128, rot=128, axes=3, mixed=True,
             adjacent=False, norm=True, packed=True, far=8192, type="bf16"),
        # A vision tower's own rotation on height and width in fp32: odd head width and row count, no norm.
        dict(name="rotate_tower_f32", op="rotate", rows=2437, hq=16, hk=16, dh=72, rot=72, axes=2, mixed=False,
             adjacent=True, norm=False, packed=False, far=64, type="f32"),
        # Training on the ragged batch: 16 sequences of about 1000 tokens, 28 query and 4 key heads.
        dict(name="grad_b16_train", op="rotate_grad", rows=16171, hq=28, hk=4, dh=128, rot=128, axes=3, mixed=True,
             adjacent=False, norm=True, packed=True, far=8192, type="bf16"),
        # A small fp16 training step, half of each head rotated.
        dict(name="grad_small_f16", op="rotate_grad", rows=333, hq=12, hk=2, dh=64, rot=32, axes=1, mixed=False,
             adjacent=False, norm=True, packed=False, far=1024, type="f16"),
        # 16 pruned prompts admitted to the cache: pages reserved, keys rotated into them beside the values, freed.
        dict(name="append_b16_prompt", op="append", fresh=True, seqs=16, t_lo=144, t_hi=256, hq=28, hk=4, dh=128,
             rot=128, axes=3, mixed=True, adjacent=False, norm=True, page=16, spare=8, far=8192, type="bf16"),
        # Eight questions on one LLaVA-NeXT image whose whole cache (all 32 layers) is kept: each takes its own 160
        # visual tokens of 2880, the system prompt's pages are shared.
        dict(name="fork_8q_n2880", op="fork", parents=1, each=8, base=35, span=2880, k=160, tail=0, layers=32, hk=8,
             dh=128, page=16, spare=64, type="bf16"),
        # Four sequences split in two (samples of one answer): full pages shared, the last part page copied.
        dict(name="fork_share_b4", op="fork", parents=4, each=1, base=0, span=0, k=0, tail=333, layers=28, hk=4,
             dh=128, page=32, spare=32, type="f16"),
        # Decoding of 64 sequences, pruned prompts and answers of different lengths.
        dict(name="attend_b64", op="attend", seqs=64, t_lo=200, t_hi=1600, hq=32, hk=8, dh=128, page=16, type="bf16"),
        # One long video dialogue: the split over one sequence.
        dict(name="attend_one_long", op="attend", seqs=1, t_lo=120001, t_hi=120001, hq=28, hk=4, dh=128, page=64,
             type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng) -> dict:
    op = rng.choice(["positions", "rotate", "rotate_grad", "append", "fork", "attend"])
    typ = rng.choice(["bf16", "bf16", "f16"])
    if op == "positions":
        hi = rng.randint(6, 40)
        lo = rng.randint(max(2, hi // 2), hi)
        frames = rng.choice([1, 1, 1, 2, 5])
        return dict(op=op, images=_log(rng, 1, 32), frames=frames, side_lo=lo, side_hi=hi,
                    D=rng.choice([2048, 3584, 4096]), k=rng.randint(1, frames * lo * lo), m_lo=1, m_hi=_log(rng, 4, 256))
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4, 7, 8])
    if op in ("rotate", "rotate_grad"):
        dh = rng.choice([64, 80, 96, 128, 128, 256, 72, 36])
        if dh in (72, 36):
            rot = dh
        else:
            rot = rng.choice([dh, dh, dh // 2])
        typ = rng.choice(["bf16", "bf16", "f16", "f32"])
        return dict(op=op, rows=_log(rng, 1, 12000), hq=hq, hk=hk, dh=dh, rot=rot, axes=rng.choice([1, 2, 3]),
                    mixed=rng.random() < 0.5, adjacent=rng.random() < 0.3, norm=rng.random() < 0.7,
                    packed=rng.random() < 0.5, far=_log(rng, 64, 1000000), type=typ)
    dh = rng.choice([64, 128, 128, 256])
    page = rng.choice([8, 16, 32, 64])
    if op == "append":
        t_hi = _log(rng, 8, 1024)
        return dict(op=op, fresh=rng.random() < 0.7, seqs=_log(rng, 1, 64), t_lo=max(1, t_hi // 3), t_hi=t_hi, hq=hq,
                    hk=hk, dh=dh, rot=dh, axes=rng.choice([1, 3]), mixed=rng.random() < 0.5,
                    adjacent=rng.random() < 0.3, norm=rng.random() < 0.7, page=page, spare=rng.randint(0, 16),
                    far=_log(rng, 64, 100000), type=typ)
    if op == "fork":
        kept = rng.random() < 0.7
        span = _log(rng, 64, 2880) if kept else 0
        return dict(op=op, parents=rng.randint(1, 4), each=rng.randint(1, 8), base=rng.randint(0, 90), span=span,
                    k=rng.randint(0, max(1, span // 6)) if kept else 0, tail=rng.randint(1, 500),
                    layers=rng.choice([2, 16, 28]), hk=rng.choice([2, 4, 8]), dh=rng.choice([64, 128]), page=page,
                    spare=rng.randint(0, 64), type=typ)
    t_hi = _log(rng, 4, 60000)
    return dict(op=op, seqs=_log(rng, 1, max(1, min(128, 200000 // t_hi))), t_lo=max(1, t_hi // rng.choice([1, 4, 50])),
                t_hi=t_hi, hq=hq, hk=hk, dh=dh, page=page, type=typ)


def draw(rng) -> dict:
    """One more case: sizes spread over the ranges, no costlier than the largest listed one."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _drawn(rng)
        if work(c)["bytes"] <= most and _bytes_held(c) <= 4e9:
            return c


# ----------------------------------------------------------------------------- sizes that a case fixes

def _sizes(case):
    """Lengths (and grids) of the case's images or sequences."""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["op"] == "positions":
        n = case["images"]
        grids = [(case["frames"], r.randint(case["side_lo"], case["side_hi"]), r.randint(case["side_lo"], case["side_hi"]))
                 for _ in range(n)]
        return grids, [r.randint(case["m_lo"], case["m_hi"]) for _ in range(n)]
    return [r.randint(case["t_lo"], case["t_hi"]) for _ in range(case["seqs"])]


def _row_counts(case):
    """append: rows of each sequence in this call, and lengths before it."""
    lens = _sizes(case)
    return (lens, [0] * len(lens)) if case["fresh"] else ([1] * len(lens), [t - 1 for t in lens])


def _parent_len(case):
    return case["base"] + case["span"] + case["tail"]


def _child_len(case):
    return case["base"] + case["k"] + case["tail"]


def _pages_of(lens, page):
    return sum(-(-t // page) for t in lens)


def _fork_new_rows(case):
    """Rows that each child needs in pages of its own."""
    shared = (case["base"] if case["span"] else _parent_len(case)) // case["page"]
    return _child_len(case) - shared * case["page"]


def _bytes_held(case):
    if case["op"] == "attend":
        return 4 * SIZE[case["type"]] * case["hk"] * case["dh"] * case["seqs"] * (case["t_hi"] + case["page"])
    if case["op"] == "fork":
        row = 2 * case["layers"] * case["hk"] * case["dh"] * 2
        return 4 * row * case["parents"] * (_parent_len(case) + case["each"] * (_child_len(case) + case["page"]))
    return 0


def work(case) -> dict:
    op = case["op"]
    if op == "positions":
        _, lens = _sizes(case)
        rows = case["images"] * case["k"] + sum(lens)
        return {"bytes": rows * (2 * case["D"] * 2 + 12) + 4 * case["images"] * case["k"], "flops": 0}
    s = SIZE[case["type"]]
    if op in ("rotate", "rotate_grad"):
        n = case["rows"] * (case["hq"] + case["hk"]) * case["dh"]
        moved = 2 if op == "rotate" or not case["norm"] else 3
        return {"bytes": n * s * moved + 4 * case["axes"] * case["rows"], "flops": n * (8 if op == "rotate" else 14)}
    if op == "append":
        rows = sum(_row_counts(case)[0])
        return {"bytes": rows * ((case["hq"] + 2 * case["hk"]) * case["dh"] * s * 2 + 4 * case["axes"] + 4),
                "flops": rows * (case["hq"] + case["hk"]) * case["dh"] * 8}
    if op == "fork":
        n = case["parents"] * case["each"]
        row = 2 * case["layers"] * case["hk"] * case["dh"] * s
        return {"bytes": n * (_fork_new_rows(case) * row * 2 + 4 * case["k"] + 8 * (-(-_child_len(case) // case["page"]))),
                "flops": 0}
    t = sum(_sizes(case))
    return {"bytes": (2 * t * case["hk"] + 2 * case["seqs"] * case["hq"]) * case["dh"] * s,
            "flops": 4 * t * case["hq"] * case["dh"]}


# ----------------------------------------------------------------------------- inputs

def _gen(seed: int) -> torch.Generator:
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 17) % (1 << 62))


def _inv_freq(rot):
    return [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]


def _axis(case):
    """The axis that turns each pair: in runs (the first pairs by time, the next by height, ...) or by turns."""
    half, axes = case["rot"] // 2, case["axes"]
    return [i % axes for i in range(half)] if case["mixed"] else [i * axes // half for i in range(half)]


def _heads(case, g, rows, typ):
    """q and k (and v): views of one projection's output, or arrays of their own."""
    hq, hk, dh = case["hq"], case["hk"], case["dh"]
    if case.get("packed", True):
        x = torch.randn(rows, (hq + 2 * hk) * dh, generator=g, device=DEV, dtype=typ)
        return (x[:, : hq * dh].view(rows, hq, dh), x[:, hq * dh: (hq + hk) * dh].view(rows, hk, dh),
                x[:, (hq + hk) * dh:].view(rows, hk, dh))
    return tuple(torch.randn(rows, h, dh, generator=g, device=DEV, dtype=typ) for h in (hq, hk, hk))


def _rotation(case, g, rows, s):
    typ, dh = TYPES[case["type"]], case["dh"]
    s["q"], s["k"], s["v"] = _heads(case, g, rows, typ)
    s["pos"] = torch.randint(0, case["far"], (case["axes"], rows), generator=g, device=DEV, dtype=torch.int32)
    s["wq"] = s["wk"] = None
    if case["norm"]:
        s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(dh, generator=g, device=DEV)).to(typ) for _ in range(2))
    s["inv_freq"], s["axis"] = _inv_freq(case["rot"]), _axis(case)
    s["inv"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device=DEV)
    s["axis_t"] = torch.tensor(s["axis"], dtype=torch.int64, device=DEV)
    if own:
        from paper_2608_06411_gb300 import binding as mb
        s["rope"] = mb.Rope(dh, s["inv_freq"], axis=s["axis"], adjacent=case["adjacent"], eps=EPS)


def _cache(case, g, layers, lens, seqs, max_pages, spare, s):
    """A pool with the first sequences' pages at random places, and its page table."""
    page, hk, dh = case["page"], case["hk"], case["dh"]
    used = [-(-t // page) for t in lens]
    pages = sum(used) + spare
    s["pool"] = torch.randn(layers, 2, pages, hk, page, dh, generator=g, device=DEV, dtype=TYPES[case["type"]])
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(seqs, max_pages, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = order[at: at + n]
        at += n
    s["table"] = table
    s["length"] = torch.zeros(seqs, dtype=torch.int32, device=DEV)
    s["length"][: len(lens)] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    s["refs"][order[:at].long()] = 1
    if own:
        from paper_2608_06411_gb300 import binding as mb
        s["cache"] = mb.Cache(s["pool"], s["table"], s["length"], s["refs"])


def prepare(case, seed) -> dict:
    g = _gen(seed)
    s = {"case": dict(case)}
    op = case["op"]
    if op == "positions":
        grids, lens = _sizes(case)
        B, D, k = case["images"], case["D"], case["k"]
        N = max(t * h * w for t, h, w in grids)
        s["grids"], s["lens"], s["N"] = grids, lens, N
        s["vis"] = torch.randn(B, N, D, generator=g, device=DEV, dtype=torch.bfloat16).view(torch.int16)
        s["text"] = torch.randn(sum(lens), D, generator=g, device=DEV, dtype=torch.bfloat16).view(torch.int16)
        r = torch.rand(B, N, generator=g, device=DEV)
        valid = torch.tensor([t * h * w for t, h, w in grids], device=DEV)
        r = torch.where(torch.arange(N, device=DEV)[None] < valid[:, None], r, torch.full_like(r, -1.0))
        s["keep"] = r.topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32)
        s["steps"] = [2] * B
        s["offset"] = 35
        if own:
            from paper_2608_06411_gb300 import binding as mb
            w = {n: torch.zeros(sh, dtype=torch.int16, device=DEV) for n, sh in
                 (("wT1", (256, D)), ("bT1", (256,)), ("wT2", (256, 256)), ("bT2", (256,)), ("wQ", (64, 256)),
                  ("wV1", (256, D)), ("bV1", (256,)), ("wV2", (256, 256)), ("bV2", (256,)), ("wK", (64, 256)))}
            s["ctx"] = mb.Context(w, D, 256, 64)
        return s
    if op in ("rotate", "rotate_grad"):
        _rotation(case, g, case["rows"], s)
        if op == "rotate_grad":
            typ = TYPES[case["type"]]
            s["dq_out"], s["dk_out"] = (torch.randn(case["rows"], h, case["dh"], generator=g, device=DEV, dtype=typ)
                                        for h in (case["hq"], case["hk"]))
        return s
    if op == "append":
        new, before = _row_counts(case)
        n, page = case["seqs"], case["page"]
        max_pages = max(-(-(a + b) // page) for a, b in zip(new, before)) + 1
        _rotation(case, g, sum(new), s)
        after = [a + b for a, b in zip(new, before)]
        if case["fresh"]:      # all pages are free
            _cache(case, g, 1, [], n, max_pages, _pages_of(after, page) + case["spare"], s)
        else:                  # the step's rows are reserved already: the last of each sequence
            _cache(case, g, 1, after, n, max_pages, case["spare"], s)
            last = torch.tensor([t - 1 for t in after], device=DEV)
            s["slots"] = s["table"][torch.arange(n, device=DEV), last // page] * page + (last % page).to(torch.int32)
        s["seqs"] = torch.arange(n, dtype=torch.int32, device=DEV)
        s["counts"] = torch.tensor(new, dtype=torch.int32, device=DEV)
        s["rows"] = sum(new)
        return s
    if op == "fork":
        par, each, page = case["parents"], case["each"], case["page"]
        n = par * each
        max_pages = -(-max(_parent_len(case), _child_len(case)) // page) + 1
        lens = [_parent_len(case)] * par
        _cache(case, g, case["layers"], lens, par + n, max_pages, n * -(-_child_len(case) // page) + case["spare"], s)
        s["parents"] = torch.arange(par, dtype=torch.int32, device=DEV).repeat_interleave(each)
        s["children"] = torch.arange(par, par + n, dtype=torch.int32, device=DEV)
        s["keep"] = s["base"] = s["span"] = None
        if case["span"]:
            s["keep"] = torch.rand(n, case["span"], generator=g, device=DEV).topk(case["k"], dim=1).indices \
                .sort(dim=1).values.to(torch.int32)
            s["base"] = torch.full((n,), case["base"], dtype=torch.int32, device=DEV)
            s["span"] = torch.full((n,), case["span"], dtype=torch.int32, device=DEV)
        return s
    lens = _sizes(case)
    n = case["seqs"]
    _cache(case, g, 1, lens, n, max(-(-t // case["page"]) for t in lens), 3, s)
    s["q"] = torch.randn(n, case["hq"], case["dh"], generator=g, device=DEV, dtype=TYPES[case["type"]]) * 2
    s["seqs"] = torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    return s


# ----------------------------------------------------------------------------- one pass

def run(s):
    return _own(s) if own else PLAIN[s["case"]["op"]](s)


def _own(s):
    op = s["case"]["op"]
    if op == "positions":
        return s["ctx"].assemble_axes(s["vis"], s["keep"], s["text"], s["lens"], s["grids"], t_step=s["steps"],
                                      pos_offset=s["offset"])
    if op == "rotate":
        return s["rope"].rotate(s["q"], s["k"], s["pos"], s["wq"], s["wk"])
    if op == "rotate_grad":
        if s["wq"] is None:
            return s["rope"].grad(s["dq_out"], s["dk_out"], s["pos"])[:2]
        return s["rope"].grad(s["dq_out"], s["dk_out"], s["pos"], s["q"], s["k"], s["wq"], s["wk"])
    c = s["cache"]
    if op == "append":
        slots = c.extend(s["seqs"], s["counts"], rows=s["rows"]) if s["case"]["fresh"] else s["slots"]
        q = s["rope"].append(s["q"], s["k"], s["v"], s["pos"], c, 0, slots, s["wq"], s["wk"])
        if s["case"]["fresh"]:
            c.free(s["seqs"])
        return q, slots, s["pool"], s["table"], s["length"], s["refs"]
    if op == "fork":
        c.fork(s["parents"], s["children"], s["keep"], s["base"], s["span"])
        c.free(s["children"])
        return s["pool"], s["table"], s["length"], s["refs"]
    return c.attend(s["q"], s["seqs"], 0)


# The plain forms: elementary torch operations in fp32 (angles in fp64), one rounding at the end.

def _plain_positions(s):
    k, N, off = s["case"]["k"], s["N"], s["offset"]
    lens = torch.tensor(s["lens"], device=DEV)
    grids = torch.tensor(s["grids"], device=DEV)
    step = torch.tensor(s["steps"], device=DEV)
    B, rows = len(s["lens"]), len(s["lens"]) * k + sum(s["lens"])
    count = lens + k
    img = torch.repeat_interleave(torch.arange(B, device=DEV), count, output_size=rows)
    j = torch.arange(rows, device=DEV) - (count.cumsum(0) - count)[img]
    tok = s["keep"][img, j.clamp(max=k - 1)].long()
    visual = j < k
    trow = ((lens.cumsum(0) - lens)[img] + j - k).clamp(min=0)
    seq = torch.where(visual[:, None], s["vis"][img, tok], s["text"][trow])
    t, h, w = grids[img].unbind(1)
    st = step[img]
    after = torch.maximum((t - 1) * st + 1, torch.maximum(h, w)) + j - k
    at = torch.stack((tok // (h * w) * st, tok // w % h, tok % w))
    return seq, (torch.where(visual, at, after) + off).to(torch.int32)


def _angles(s):
    a = s["pos"].double()[s["axis_t"]].T * s["inv"]                       # [rows, rot / 2]
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _split(x, rot, adjacent):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., : rot // 2], x[..., rot // 2: rot])


def _turn(x, cos, sin, rot, adjacent):
    a, b = _split(x, rot, adjacent)
    lo, hi = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((lo, hi), -1).flatten(-2) if adjacent else torch.cat((lo, hi), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _normed(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _plain_rotate(s):
    c, out = s["case"], []
    cos, sin = _angles(s)
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.float() if w is None else _normed(x.float(), w)
        out.append(_turn(y, cos, sin, c["rot"], c["adjacent"]).to(x.dtype))
    return tuple(out)


def _plain_rotate_grad(s):
    c, dx, dw = s["case"], [], []
    cos, sin = _angles(s)
    for x, w, dy in ((s["q"], s["wq"], s["dq_out"]), (s["k"], s["wk"], s["dk_out"])):
        g = _turn(dy.float(), cos, -sin, c["rot"], c["adjacent"])
        if w is not None:
            xf = x.float()
            r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
            xn = xf * r
            dw.append((g * xn).sum((0, 1), dtype=torch.float64).float())
            gw = g * w.float()
            g = r * (gw - xn * (gw * xn).mean(-1, keepdim=True))
        dx.append(g.to(dy.dtype))
    return tuple(dx + dw)


def _free_pages(refs):
    """Page numbers, the free ones first, in ascending order."""
    return torch.argsort((refs > 0).to(torch.uint8), stable=True)


def _release(s, seqs):
    page = s["case"]["page"]
    seqs = seqs.long()
    n = (s["length"][seqs] + page - 1) // page
    on = torch.arange(s["table"].shape[1], device=DEV)[None] < n[:, None]
    s["refs"].index_add_(0, s["table"][seqs].flatten(), -on.flatten().to(torch.int32))
    s["length"][seqs] = 0


def _plain_append(s):
    c, page = s["case"], s["case"]["page"]
    if c["fresh"]:
        seqs, new = s["seqs"].long(), s["counts"]
        before = s["length"][seqs]
        have, want = (before + page - 1) // page, (before + new + page - 1) // page
        col = torch.arange(s["table"].shape[1], device=DEV)[None]
        on = (col >= have[:, None]) & (col < want[:, None])
        first = (want - have).cumsum(0) - (want - have)
        free = _free_pages(s["refs"])
        got = free[(first[:, None] + col - have[:, None]).clamp(0, free.numel() - 1)].to(torch.int32)
        s["table"][seqs] = torch.where(on, got, s["table"][seqs])
        s["refs"].index_add_(0, s["table"][seqs].flatten(), on.flatten().to(torch.int32))
        s["length"][seqs] = before + new
        i = torch.repeat_interleave(torch.arange(len(seqs), device=DEV), new, output_size=s["rows"])
        t = before[i] + torch.arange(s["rows"], device=DEV) - (new.cumsum(0) - new)[i]
        slots = (s["table"][seqs[i], t // page] * page + t % page).to(torch.int32)
    else:
        slots = s["slots"]
    q, k = _plain_rotate(s)
    p, o = (slots // page).long(), (slots % page).long()
    s["pool"][0, 0][p, :, o] = k
    s["pool"][0, 1][p, :, o] = s["v"]
    if c["fresh"]:
        _release(s, s["seqs"])
    return q, slots, s["pool"], s["table"], s["length"], s["refs"]


def _plain_fork(s):
    c, page = s["case"], s["case"]["page"]
    par, chi = s["parents"].long(), s["children"].long()
    was = s["length"][par].long()
    if s["keep"] is None:
        base, span, k, shared, new = was, torch.zeros_like(was), 0, was // page, was
    else:
        base, span, k = s["base"].long(), s["span"].long(), c["k"]
        shared, new = base // page, was - span + k
    want = (new + page - 1) // page
    col = torch.arange(s["table"].shape[1], device=DEV)[None]
    first = (want - shared).cumsum(0) - (want - shared)
    free = _free_pages(s["refs"])
    got = free[(first[:, None] + col - shared[:, None]).clamp(0, free.numel() - 1)].to(torch.int32)
    on = col < want[:, None]
    row = torch.where(col < shared[:, None], s["table"][par], torch.where(on, got, s["table"][chi]))
    s["table"][chi] = row
    s["refs"].index_add_(0, row.flatten(), on.flatten().to(torch.int32))
    s["length"][chi] = new.to(torch.int32)
    j = torch.arange(_child_len(c), device=DEV)[None]
    src = torch.where(j < base[:, None], j, j - k + span[:, None])
    if k:
        kept = s["keep"].gather(1, (j - base[:, None]).clamp(0, k - 1)).long() + base[:, None]
        src = torch.where((j >= base[:, None]) & (j < base[:, None] + k), kept, src)
    i, t = torch.nonzero((j >= (shared * page)[:, None]) & (j < new[:, None]), as_tuple=True)
    f = src[i, t]
    sp, so = s["table"][par[i], f // page].long(), f % page
    dp, do = row[i, t // page].long(), t % page
    pool = s["pool"].flatten(0, 1)
    pool[:, dp, :, do] = pool[:, sp, :, so]
    _release(s, s["children"])
    return s["pool"], s["table"], s["length"], s["refs"]


def _plain_attend(s):
    page, q = s["case"]["page"], s["q"].float()
    seqs = s["seqs"].long()
    n, hq, dh = q.shape
    pages = s["table"][seqs].long()
    k, v = (s["pool"][0, i][pages].transpose(2, 3).flatten(1, 2).float() for i in (0, 1))      # [n, tokens, hk, dh]
    hk = k.shape[2]
    on = torch.arange(k.shape[1], device=DEV)[None] < s["length"][seqs][:, None]
    v = torch.where(on[:, :, None, None], v, torch.zeros_like(v))
    z = torch.einsum("nhgd,nthd->nhgt", q.view(n, hk, hq // hk, dh), k) / math.sqrt(dh)
    z = torch.where(on[:, None, None], z, torch.full_like(z, -math.inf))
    e = torch.exp(z - z.amax(-1, keepdim=True))
    o = torch.einsum("nhgt,nthd->nhgd", e / e.sum(-1, keepdim=True), v)
    return o.reshape(n, hq, dh).to(s["q"].dtype)


PLAIN = {"positions": _plain_positions, "rotate": _plain_rotate, "rotate_grad": _plain_rotate_grad,
         "append": _plain_append, "fork": _plain_fork, "attend": _plain_attend}


# ----------------------------------------------------------------------------- 64-bit values

def _def_rotate(x, w, pos, inv_freq, axis, adjacent):
    """x [rows, heads, dh] in fp64: the head over its root mean square, times w; pair i turned as a complex number."""
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
    half = len(inv_freq)
    turn = torch.stack([torch.polar(torch.ones_like(pos[0], dtype=torch.float64), pos[axis[i]].double() * inv_freq[i])
                        for i in range(half)], 1)[:, None]
    head = x[..., : 2 * half].unflatten(-1, (half, 2) if adjacent else (2, half))
    z = torch.complex(head.select(-1 if adjacent else -2, 0), head.select(-1 if adjacent else -2, 1)) * turn
    y = torch.stack((z.real, z.imag), -1 if adjacent else -2).flatten(-2)
    return torch.cat((y, x[..., 2 * half:]), -1)


def _exact_rotate(s):
    return [_def_rotate(x.double(), None if w is None else w.double(), s["pos"], s["inv_freq"], s["axis"],
                        s["case"]["adjacent"]) for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"]))]


def exact(case, seed):
    s = prepare(case, seed)
    op, page = case["op"], case.get("page", 1)
    if op == "positions":
        rows, ids, at = [], [], 0
        keep = s["keep"].cpu().numpy()
        for b, ((T, H, W), m) in enumerate(zip(s["grids"], s["lens"])):
            st = s["steps"][b]
            rows += [s["vis"][b][s["keep"][b].long()], s["text"][at: at + m]]
            ids += [(n // (H * W) * st, n % (H * W) // W, n % W) for n in keep[b].tolist()]
            ids += [(max((T - 1) * st + 1, H, W) + i,) * 3 for i in range(m)]
            at += m
        return torch.cat(rows), torch.from_numpy(np.array(ids, np.int64).T.astype(np.int32) + np.int32(s["offset"]))
    if op == "rotate":
        return tuple(_exact_rotate(s))
    if op == "rotate_grad":
        dx, dw = [], []
        for x, w, dy in ((s["q"], s["wq"], s["dq_out"]), (s["k"], s["wk"], s["dk_out"])):
            x = x.double().requires_grad_()
            w = None if w is None else w.double().requires_grad_()
            y = _def_rotate(x, w, s["pos"], s["inv_freq"], s["axis"], case["adjacent"])
            got = torch.autograd.grad(y, [x] if w is None else [x, w], dy.double())
            dx.append(got[0])
            dw += got[1:]
        return tuple(dx + dw)
    pool, table = s["pool"], s["table"].cpu().numpy()
    lens, refs = s["length"].cpu().numpy(), s["refs"].cpu().numpy()
    if op == "append":
        q, k = _exact_rotate(s)
        new = s["counts"].tolist()
        if case["fresh"]:
            free = [p for p in range(len(refs)) if refs[p] == 0]
            slots = []
            for i, n in enumerate(new):
                for t in range(n):
                    if t % page == 0:
                        table[i, t // page] = free.pop(0)
                    slots.append(int(table[i, t // page]) * page + t % page)
        else:
            slots = [int(table[i, (lens[i] - 1) // page]) * page + (lens[i] - 1) % page for i in range(len(new))]
        wide = pool.double()
        for r, sl in enumerate(slots):
            wide[0, 0, sl // page, :, sl % page] = k[r]
            wide[0, 1, sl // page, :, sl % page] = s["v"][r].double()
        return q, torch.tensor(slots, dtype=torch.int32), wide, torch.from_numpy(table), s["length"], s["refs"]
    if op == "fork":
        before = pool.clone()
        free = [p for p in range(len(refs)) if refs[p] == 0]
        for i, (p, c) in enumerate(zip(s["parents"].tolist(), s["children"].tolist())):
            src = list(range(lens[p]))
            shared = len(src) // page
            if case["span"]:
                b = case["base"]
                src = src[:b] + [b + int(t) for t in s["keep"][i].tolist()] + src[b + case["span"]:]
                shared = b // page
            for t0 in range(0, len(src), page):
                if t0 // page < shared:
                    table[c, t0 // page] = table[p, t0 // page]
                    continue
                to = free.pop(0)
                table[c, t0 // page] = to
                for o, f in enumerate(src[t0: t0 + page]):
                    pool[:, :, to, :, o] = before[:, :, int(table[p, f // page]), :, f % page]
        return pool, torch.from_numpy(table), s["length"], s["refs"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for i, b in enumerate(s["seqs"].tolist()):
        n = int(lens[b])
        at = torch.from_numpy(table[b, : -(-n // page)].astype(np.int64)).to(DEV)
        k, v = (pool[0, j][at].double().permute(1, 0, 2, 3).flatten(1, 2)[:, :n] for j in (0, 1))
        g = case["hq"] // case["hk"]
        for h in range(case["hq"]):
            p = torch.softmax(k[h // g] @ s["q"][i, h].double() / math.sqrt(case["dh"]), 0)
            out[i, h] = p @ v[h // g]
    return out
