"""Plain 64-bit models of the language-model hand-off (numpy): positions on axes, the per-head norm with rotation and
its gradient, the pages of a cache as Python lists, and attention of single tokens."""
from __future__ import annotations

import numpy as np


def axis_positions(keep, lens, grids, t_step=None, pos_offset=0):
    """Position ids [3, rows] of map_assemble_axes, token by token."""
    out = []
    for b, (T, H, W) in enumerate(grids):
        st = 1 if t_step is None else int(t_step[b])
        for n in keep[b]:
            n = int(n)
            out.append((n // (H * W) * st, n % (H * W) // W, n % W))
        nxt = max((T - 1) * st + 1, H, W)
        out += [(nxt + m,) * 3 for m in range(int(lens[b]))]
    return (np.array(out, dtype=np.int64).reshape(-1, 3) + pos_offset).T.astype(np.int32)


def pairs_of(rot, adjacent):
    half = rot // 2
    return (2 * np.arange(half), 2 * np.arange(half) + 1) if adjacent else (np.arange(half), np.arange(half) + half)


def rotate(x, w, pos, inv_freq, axis, adjacent, eps):
    """x [rows, heads, dh] float64 -> (y, z): z the normed head, y the rotated one."""
    z = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y = z.copy()
    a, b = pairs_of(2 * len(inv_freq), adjacent)
    if len(inv_freq):
        ang = np.asarray(pos, np.float64)[np.asarray(axis)].T * np.asarray(inv_freq, np.float64)   # [rows, half]
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        y[..., a] = z[..., a] * c - z[..., b] * s
        y[..., b] = z[..., b] * c + z[..., a] * s
    return y, z


def rotate_grad(dy, x, w, pos, inv_freq, axis, adjacent, eps):
    """(dx, dw): the chain rule written out; dw None without a norm."""
    g = rotate(dy, None, pos, -np.asarray(inv_freq, np.float64), axis, adjacent, eps)[0]
    if w is None:
        return g, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdims=True))
    return dx, (g * n).sum((0, 1))


class Pages:
    """A cache as lists: rows[s] = the slots of sequence s; the lowest free pages are taken first."""

    def __init__(self, pages, page, seqs, max_pages):
        self.page, self.max_pages = page, max_pages
        self.table = [[] for _ in range(seqs)]
        self.length = [0] * seqs
        self.refs = [0] * pages

    def _free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def extend(self, seqs, counts, rows):
        """Slots [rows], or None if the call is refused; counts None: entry i has row i."""
        if counts is None:
            real = [i for i, s in enumerate(seqs) if s != -1]
            got = self.extend([seqs[i] for i in real], [1] * len(real), len(real)) if len(seqs) <= rows else None
            if got is None:
                return None
            out = [-1] * rows
            for i, s in zip(real, got):
                out[i] = s
            return out
        named = [s for s in seqs if s != -1]
        if len(set(named)) < len(named) or any(s < 0 or s >= len(self.table) for s in named):
            return None
        add = [0 if s == -1 else c for s, c in zip(seqs, counts)]
        if any(c < 0 for c in add) or sum(add) > rows:
            return None
        free, plan = self._free(), []
        for s, c in zip(seqs, add):
            need = -(-(self.length[s] + c) // self.page) - len(self.table[s]) if s != -1 else 0
            if s != -1 and len(self.table[s]) + need > self.max_pages or need > len(free):
                return None
            plan.append(free[:need])
            free = free[need:]
        slots = []
        for s, c, got in zip(seqs, add, plan):
            if s == -1:
                continue
            self.table[s] += got
            for p in got:
                self.refs[p] = 1
            for t in range(self.length[s], self.length[s] + c):
                slots.append(self.table[s][t // self.page] * self.page + t % self.page)
            self.length[s] += c
        return slots + [-1] * (rows - len(slots))

    def slots(self, s):
        return [self.table[s][t // self.page] * self.page + t % self.page for t in range(self.length[s])]

    def fork(self, parents, children, keep=None, base=None, span=None):
        """[(slot, source slot or -1 for a bad index)] of the copied rows, or None if the call is refused."""
        n = len(self.table)
        if any(p < 0 or p >= n for p in parents) or any(c < 0 or c >= n or self.length[c] for c in children):
            return None
        if len(set(children)) < len(children) or set(children) & set(parents):
            return None
        free, plan = self._free(), []
        for i, (p, c) in enumerate(zip(parents, children)):
            src, shared = list(range(self.length[p])), self.length[p] // self.page
            if base is not None:
                b, sp = base[i], span[i]
                if b < 0 or sp < 0 or b + sp > len(src):
                    return None
                kept = [] if keep is None else [b + x if 0 <= x < sp else -1 for x in keep[i]]
                src, shared = src[:b] + kept + src[b + sp:], b // self.page
            want = -(-len(src) // self.page)
            if want > self.max_pages or want - shared > len(free):
                return None
            plan.append((src, self.table[p][:shared], free[: want - shared]))
            free = free[want - shared:]
        copies = []
        for (src, shared, got), p, c in zip(plan, parents, children):
            self.table[c], self.length[c] = shared + got, len(src)
            for x in shared + got:
                self.refs[x] += 1
            at = self.slots(p)
            copies += [(self.table[c][t // self.page] * self.page + t % self.page, -1 if f < 0 else at[f])
                       for t, f in enumerate(src) if t >= len(shared) * self.page]
        return copies

    def free(self, seqs):
        for s in seqs:
            if s == -1:
                continue
            for p in self.table[s]:
                self.refs[p] -= 1
            self.table[s], self.length[s] = [], 0


def attend(q, k, v, scale):
    """q [heads, dh], k and v [rows, kv heads, dh] float64 -> (out, sum p |v|, largest sum |q k| scale)."""
    g = q.shape[0] // k.shape[1]
    out, mag, dz = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for h in range(q.shape[0]):
        if not k.shape[0]:
            continue
        z = k[:, h // g] @ q[h] * scale
        p = np.exp(z - z.max())
        p /= p.sum()
        out[h], mag[h] = p @ v[:, h // g], p @ np.abs(v[:, h // g])
        dz = max(dz, float((np.abs(k[:, h // g]) @ np.abs(q[h])).max() * abs(scale)))
    return out, mag, dz
