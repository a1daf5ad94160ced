"""The cache of a live view, its attention and rotary positions with several
axes, plainly: lists, numpy and 64 bits.

The page operators follow their rules one entry at a time: every entry reads
the state before the call, new pages are the lowest-numbered free ones in
entry order, pages given back are free from the next call on, a malformed
entry or one that finds too few pages changes nothing and is counted.
"""
from __future__ import annotations

import math

import numpy as np


class Cache:
    def __init__(self, layers, pages, page, heads, d, seqs, max_pages):
        self.page, self.max_pages, self.n_seqs, self.n_pages = page, max_pages, seqs, pages
        self.k = np.zeros((layers, pages, heads, page, d))
        self.v = np.zeros((layers, pages, heads, page, d))
        self.table = [[] for _ in range(seqs)]
        self.len = [0] * seqs
        self.refs = [0] * pages
        self.no_pages = self.bad = 0

    # what the device arrays hold
    def page_table(self):
        return np.array([t + [-1] * (self.max_pages - len(t)) for t in self.table], dtype=np.int32)

    def free_pages(self):
        return sum(r == 0 for r in self.refs)

    def rows(self, s):
        """(page, place) of every row of sequence s."""
        return [(self.table[s][r // self.page], r % self.page) for r in range(self.len[s])]

    def gather(self, layer, s):
        at = self.rows(s)
        pick = lambda x: (np.stack([x[layer, p, :, r] for p, r in at]) if at
                          else np.zeros((0,) + x.shape[2:3] + x.shape[4:]))
        return pick(self.k), pick(self.v)

    def _deal(self, needs):
        """Pages of each entry, or None from where they do not suffice."""
        free = [p for p, r in enumerate(self.refs) if r == 0]
        out, asked = [], 0
        for n in needs:
            asked += n
            out.append(free[asked - n:asked] if n == 0 or asked <= len(free) else None)
        return out

    def reserve(self, ids, ptr, n_new):
        slot, pos = [-1] * n_new, [-1] * n_new
        seen, want = set(), []
        for e, s in enumerate(ids):
            a, b = ptr[e], ptr[e + 1]
            inside = 0 <= s < self.n_seqs
            bad = a < 0 or b < a or b > n_new or (not inside and s != -1) or s in seen
            if inside:
                seen.add(s)
            if bad:
                self.bad += 1
            if bad or not inside:
                want.append(None)
                continue
            total = -(-(self.len[s] + b - a) // self.page)
            if total > self.max_pages:
                self.no_pages += 1
                want.append(None)
            else:
                want.append((s, a, b - a, total - len(self.table[s])))
        dealt = self._deal([w[3] if w else 0 for w in want])
        for w, pages in zip(want, dealt):
            if w is None:
                continue
            s, a, n, _ = w
            if pages is None:
                self.no_pages += 1
                continue
            self.table[s] += pages
            for p in pages:
                self.refs[p] = 1
            for i in range(n):
                r = self.len[s] + i
                slot[a + i] = self.table[s][r // self.page] * self.page + r % self.page
                pos[a + i] = r
            self.len[s] += n
        return slot, pos

    def write(self, layer, slot, k, v):
        for i, x in enumerate(slot):
            if 0 <= x < self.n_pages * self.page:
                self.k[layer, x // self.page, :, x % self.page] = k[i]
                self.v[layer, x // self.page, :, x % self.page] = v[i]

    def free(self, ids):
        done = set()
        for s in ids:
            if not 0 <= s < self.n_seqs:
                self.bad += s != -1
            elif s not in done:
                done.add(s)
                for p in self.table[s]:
                    self.refs[p] -= 1
                self.table[s], self.len[s] = [], 0

    def fork(self, src, dst, share=True):
        self._move(src, dst, None, share)

    def compact(self, src, dst, spans):
        self._move(src, dst, spans, True)

    def _move(self, src, dst, spans, share):
        inside = lambda s: 0 <= s < self.n_seqs
        in_place = {s for s, t in zip(src, dst) if s == t and spans is not None}
        named, plan = set(), []
        for e, (s, t) in enumerate(zip(src, dst)):
            ok = inside(s) and inside(t) and t not in named
            if inside(t):
                named.add(t)
            if ok and s != t:
                ok = self.len[t] == 0 and s not in in_place
            if spans is None:
                ok = ok and s != t
            cut = list(spans[e]) if spans is not None else []
            at = 0
            for a, b in cut:
                ok = ok and at <= a <= b
                at = b
            if not ok:
                self.bad += 1
                plan.append(None)
                continue
            n = self.len[s]
            gone = {r for a, b in cut for r in range(min(a, n), min(b, n))}
            rows = [r for r in range(n) if r not in gone]
            first = min(gone) if gone else n
            keep = first // self.page if share or s == t else 0
            if s == t and first == len(rows) and first % self.page \
                    and self.refs[self.table[s][keep]] == 1:
                keep += 1
            plan.append((s, t, rows, keep, -(-len(rows) // self.page) - keep))
        dealt = self._deal([p[4] if p else 0 for p in plan])
        old = [list(t) for t in self.table]
        refs = list(self.refs)
        for p, pages in zip(plan, dealt):
            if p is None:
                continue
            s, t, rows, keep, n = p
            if pages is None:
                self.no_pages += 1
                continue
            for i in range(keep * self.page, len(rows)):
                a, b = old[s][rows[i] // self.page], rows[i] % self.page
                x, y = pages[i // self.page - keep], i % self.page
                self.k[:, x, :, y] = self.k[:, a, :, b]
                self.v[:, x, :, y] = self.v[:, a, :, b]
            for q in pages:
                refs[q] += 1
            if s == t:
                for q in old[s][keep:]:
                    refs[q] -= 1
            else:
                for q in old[s][:keep]:
                    refs[q] += 1
            self.table[t], self.len[t] = old[s][:keep] + pages, len(rows)
        self.refs = refs


def tree_rows(parent, n):
    """[n, n] bool and depths: a row and its ancestors (parents come before their children)."""
    see, depth = np.zeros((n, n), dtype=bool), []
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            j = parent[j] if parent[j] < j else -1
        depth.append(int(see[i].sum()) - 1)
    return see, depth


def attend(k, v, q, see, scale):
    """Attention of q [n, hq, d] over k, v [L, hkv, d] with see [n, L]: o, lse
    [hq, n], and sum |weight v| (what a relative error of the weights scales).
    A row that sees nothing: 0, -inf.  Unseen rows are left out, not multiplied by 0."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    o, lse, mag = np.zeros(q.shape), np.full((hq, n), -math.inf), np.zeros(q.shape)
    for i in range(n):
        j = np.flatnonzero(see[i])
        if not len(j):
            continue
        for h in range(hq):
            z = (k[j, h // g] @ q[i, h]) * scale
            m = z.max()
            e = np.exp(z - m)
            w = e / e.sum()
            o[i, h], mag[i, h] = w @ v[j, h // g], w @ np.abs(v[j, h // g])
            lse[h, i] = m + math.log(e.sum())
    return o, lse, mag


def rotate(x, pos, axis, theta, inverse=False):
    """x [n, heads, d]: pair (i, i + P), P = len(axis), by pos[axis[i]] * theta^(-i/P)."""
    P = len(axis)
    y = np.array(x, dtype=np.float64)
    for i in range(P):
        a = np.asarray(pos[axis[i]], dtype=np.float64) * theta ** (-i / P)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None] * (-1 if inverse else 1)
        u, w = y[..., i].copy(), y[..., i + P].copy()
        y[..., i], y[..., i + P] = u * c - w * s, w * c + u * s
    return y
