"""Calls of the cache side of a live view, as cases that can be timed and checked.

The cache holds, page by page, the keys and values of the tokens that are live
in a context: an edit compacts it, branches and samples fork it, and rows
(single tokens, trees of drafted tokens, chunks of a prompt) attend over it.
With it go rotary positions with several axes, for rows that carry positions
of their own.  ``run`` computes each case in plain torch operations, or, with
``own`` set, through the binding ``paper_2609_00865_amd.mv``; ``exact`` gives
the same results in 64 bits, written apart from both."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
THETA = 1e6
INF = (1 << 31) - 1


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def listed():
    return [
        # One rollout decodes one token: the smallest attention call, where
        # launches and latency count.
        {"name": "decode_one", "kind": "attn", "seqs": 1, "lo": 777, "hi": 777, "rows_lo": 1,
         "rows_hi": 1, "tree": False, "hq": 28, "hkv": 4, "d": 128, "page": 16},
        # A batch of rollouts, each decoding one token over its own live
        # context of 257 to 16384 tokens.
        {"name": "decode_batch", "kind": "attn", "seqs": 64, "lo": 257, "hi": 16384,
         "rows_lo": 1, "rows_hi": 1, "tree": False, "hq": 28, "hkv": 4, "d": 128, "page": 16},
        # Few rollouts with very long contexts, 64/8 heads: the work of one
        # row has to be split along its keys.
        {"name": "decode_long", "kind": "attn", "seqs": 6, "lo": 65536, "hi": 131071,
         "rows_lo": 1, "rows_hi": 1, "tree": False, "hq": 64, "hkv": 8, "d": 128, "page": 64},
        # Trees of drafted tokens of uneven size, verified over their contexts.
        {"name": "verify_trees", "kind": "attn", "seqs": 24, "lo": 301, "hi": 8192,
         "rows_lo": 8, "rows_hi": 61, "tree": True, "hq": 28, "hkv": 4, "d": 128, "page": 16},
        # The same for a small policy with heads of 64.
        {"name": "verify_small_heads", "kind": "attn", "seqs": 9, "lo": 97, "hi": 4096,
         "rows_lo": 5, "rows_hi": 33, "tree": True, "hq": 8, "hkv": 2, "d": 64, "page": 32},
        # A chunk of a long prompt (or of a trajectory that is scored chunk by
        # chunk) over what the cache holds already: many rows, the products bound it.
        {"name": "chunk", "kind": "attn", "seqs": 2, "lo": 4099, "hi": 8192, "rows_lo": 1531,
         "rows_hi": 2048, "tree": False, "hq": 28, "hkv": 4, "d": 128, "page": 16},
        # Sampling a group of 16 rollouts from each of two prompts: the prompt's
        # pages are shared, each sample gets its own last page.
        {"name": "fork_group", "kind": "fork", "groups": 2, "children": 16, "length": 4091,
         "layers": 8, "hkv": 4, "d": 128, "page": 16},
        # An agent's fold: several runs of one long context are evicted; what
        # follows the first moves up, in place.
        {"name": "edit_in_place", "kind": "edit", "seqs": 1, "length": 32768, "spans": 16,
         "layers": 8, "hkv": 4, "d": 128, "page": 16, "in_place": True},
        # The branch that an edit opens, beside the one that goes on without it,
        # for a few rollouts.
        {"name": "edit_branch", "kind": "edit", "seqs": 5, "length": 2903, "spans": 4,
         "layers": 4, "hkv": 2, "d": 64, "page": 32, "in_place": False},
        # Q and K of one decoding step, rotated where the projection left them.
        {"name": "rope_step", "kind": "rope", "tokens": 64, "hq": 28, "hkv": 4, "d": 128,
         "rot": 128, "axes": 3, "layout": "sections", "fused": True, "both": False},
        # Q and K of a training batch of rollouts with images, and the
        # gradients rotated back.
        {"name": "rope_train", "kind": "rope", "tokens": 32768, "hq": 28, "hkv": 4, "d": 128,
         "rot": 128, "axes": 3, "layout": "interleaved", "fused": True, "both": True},
        # One verification step of a small policy as it is used: room for the drafted
        # rows, K rotated into the pages, Q rotated, attention in every layer,
        # and the accepted path kept as the context that goes on.
        {"name": "draft_step", "kind": "step", "seqs": 16, "lo": 301, "hi": 4096, "rows_lo": 6,
         "rows_hi": 24, "layers": 4, "hq": 16, "hkv": 4, "d": 128, "page": 16},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(1, 1), (8, 2), (16, 4), (28, 4), (32, 8), (12, 12), (64, 8), (16, 1)]


def draw(rng):
    kind = rng.choice(["decode", "decode", "verify", "verify", "chunk", "fork", "edit", "edit",
                       "rope", "rope", "step"])
    hq, hkv = rng.choice(HEADS)
    c = {"hq": hq, "hkv": hkv, "d": rng.choice([64, 128, 128]), "page": rng.choice([16, 16, 32, 64, 128])}
    if kind == "decode":
        seqs = _log(rng, 1, 128)
        hi = _log(rng, 64, min(131072, 1048576 // (seqs * hkv)))
        return {"kind": "attn", "seqs": seqs, "lo": _log(rng, 1, hi), "hi": hi, "rows_lo": 1,
                "rows_hi": 1, "tree": False, **c}
    if kind == "verify":
        seqs, hi = _log(rng, 1, 48), _log(rng, 64, 8192)
        top = _log(rng, 2, 96)
        return {"kind": "attn", "seqs": seqs, "lo": _log(rng, 1, hi), "hi": hi,
                "rows_lo": rng.randint(1, top), "rows_hi": top, "tree": True, **c}
    if kind == "chunk":
        seqs, hi = rng.randint(1, 3), _log(rng, 64, 8192)
        top = _log(rng, 97, 2048)
        return {"kind": "attn", "seqs": seqs, "lo": _log(rng, 1, hi), "hi": hi,
                "rows_lo": rng.randint(max(1, top // 3), top), "rows_hi": top, "tree": False,
                **{**c, "hq": min(hq, 32), "hkv": min(hkv, 4) if hq > 12 else hkv}}
    del c["hq"]
    if kind == "fork":
        return {"kind": "fork", "groups": rng.randint(1, 4), "children": rng.choice([2, 4, 8, 16]),
                "length": _log(rng, 5, 4096), "layers": rng.randint(1, 8), **c}
    if kind == "edit":
        return {"kind": "edit", "seqs": rng.randint(1, 6), "length": _log(rng, 40, 8192),
                "spans": rng.randint(1, 16), "layers": rng.randint(1, 6),
                "in_place": rng.random() < 0.5, **c}
    if kind == "rope":
        d = rng.choice([64, 80, 96, 128, 256])
        return {"kind": "rope", "tokens": _log(rng, 1, 32768) if d < 256 else _log(rng, 1, 8192),
                "hq": min(hq, 32), "hkv": min(hkv, 8), "d": d, "rot": rng.choice([d, d, d // 2]),
                "axes": rng.choice([1, 2, 3, 3, 4]),
                "layout": rng.choice(["sections", "interleaved"]),
                "fused": rng.random() < 0.6, "both": rng.random() < 0.5}
    hq, hkv = rng.choice([(8, 2), (16, 4), (28, 4), (32, 8)])
    hi, top = _log(rng, 64, 4096), rng.randint(2, 32)
    return {"kind": "step", "seqs": _log(rng, 1, 24), "lo": _log(rng, 1, hi), "hi": hi,
            "rows_lo": rng.randint(1, top), "rows_hi": top, "layers": rng.randint(1, 4),
            **c, "hq": hq, "hkv": hkv}


# --------------------------------------------------------------------------
# sizes that follow from a case alone
# --------------------------------------------------------------------------
def _spread(n, lo, hi, phase):
    """n whole numbers in [lo, hi], spread over their logarithm, the largest among them."""
    if n == 1:
        return [hi]
    f = [(phase + i * 0.6180339887498949) % 1.0 for i in range(n)]
    top = max(f)
    return [max(lo, min(hi, int(round(lo * (hi / lo) ** (x / top))))) for x in f]


def _sizes(c):
    """Context rows and new rows of every sequence."""
    return _spread(c["seqs"], c["lo"], c["hi"], 0.37), _spread(c["seqs"], c["rows_lo"],
                                                               c["rows_hi"], 0.81)


def _axis_map(pairs, axes, layout):
    """The position axis of every rotated pair: runs (the first axis a quarter,
    the others equal parts of the rest), or the axes taken in turn."""
    if layout == "interleaved":
        return [i % axes for i in range(pairs)]
    if axes == 1:
        return [0] * pairs
    first = pairs // 4
    rest, others = pairs - first, axes - 1
    sizes = [first] + [rest * (j + 1) // others - rest * j // others for j in range(others)]
    return [a for a, n in enumerate(sizes) for _ in range(n)]


def _spans(c, seed, i):
    """The evicted runs of sequence i of an edit: sorted, disjoint, about 40 %
    of the rows after the first sixteenth (the prompt stays)."""
    n, k = c["length"] - 13 * i, c["spans"]
    n = max(n, 8)
    rng = np.random.default_rng([seed, i, 5])
    lo = n // 16
    k = min(k, max(1, (n - lo) // 4))
    total = max(k, int(0.4 * (n - lo)))
    gaps_total = n - lo - total
    cut = lambda t: np.diff(np.concatenate(([0], np.sort(rng.integers(0, t + 1, k)), [t])))
    runs = 1 + cut(total - k)[:k]
    gaps = cut(max(0, gaps_total))
    out, at = [], lo
    for j in range(k):
        at += int(gaps[j])
        out.append((at, min(n, at + int(runs[j]))))
        at = out[-1][1]
    return n, out


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * salt + int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _pool(g, *shape):
    """A pool of pages, every row of it written at some time before."""
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    for layer in out:
        layer.normal_(generator=g)
    return out


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class _Book:
    """A cache as plain torch and lists: pools, page table, lengths and the
    number of sequences that hold each page."""

    def __init__(self, seed, lens, slots, spare, layers, hkv, d, page):
        self.page = page
        need = [-(-n // page) for n in lens]
        pages = sum(need) + spare
        # after some time of use a sequence's pages lie anywhere
        order = np.random.default_rng([seed, 11]).permutation(pages).tolist()
        self.width = max(need + [1]) + -(-256 // page)   # room for rows to come
        self.table, self.lens, self.refs = [], list(lens), [0] * pages
        for n in need:
            self.table.append([order.pop() for _ in range(n)])
            for p in self.table[-1]:
                self.refs[p] = 1
        for _ in range(slots - len(lens)):
            self.table.append([])
            self.lens.append(0)
        g = _gen(seed, 21)
        self.k = _pool(g, layers, pages, hkv, page, d)
        self.v = _pool(g, layers, pages, hkv, page, d)

    def tensors(self):
        rows = [t + [-1] * (self.width - len(t)) for t in self.table]
        return _i32(rows), _i32(self.lens), _i32(self.refs)

    def open(self):
        """The same state as the library's cache."""
        from paper_2609_00865_amd import mv
        layers, pages, hkv, page, d = self.k.shape
        cache = mv.PagedCache(layers, pages, page, hkv, d, len(self.table), self.width,
                              device=DEV)
        cache.k.copy_(self.k)
        cache.v.copy_(self.v)
        cache.restore(*self.tensors())
        del self.k, self.v
        return cache

    # the page operators, in lists and indexing ------------------------------
    def places(self, s, rows):
        t, p = self.table[s], self.page
        return _i64([t[r // p] for r in rows]), _i64([r % p for r in rows])

    def lowest(self, n, taken):
        out = []
        for i, r in enumerate(self.refs):
            if len(out) == n:
                break
            if r == 0 and i not in taken:
                out.append(i)
        taken.update(out)
        return out

    def reserve(self, seqs, rows):
        slot, pos, taken = [], [], set()
        for s, n in zip(seqs, rows):
            have, want = len(self.table[s]), -(-(self.lens[s] + n) // self.page)
            self.table[s] += self.lowest(want - have, taken)
            for r in range(self.lens[s], self.lens[s] + n):
                slot.append(self.table[s][r // self.page] * self.page + r % self.page)
                pos.append(r)
            self.lens[s] += n
        for p in taken:
            self.refs[p] = 1
        return slot, pos

    def free(self, seqs):
        for s in seqs:
            for p in self.table[s]:
                self.refs[p] -= 1
            self.table[s], self.lens[s] = [], 0

    def compact(self, srcs, dsts, spans):
        p, taken, plan = self.page, set(), []
        for s, t, cut in zip(srcs, dsts, spans):
            n = self.lens[s]
            cut = [(min(a, n), min(b, n)) for a, b in cut]
            cut = [x for x in cut if x[1] > x[0]]
            first = cut[0][0] if cut else n
            rows, at = [], 0
            for a, b in cut + [(n, n)]:
                rows += range(at, a)
                at = b
            kept = first // p
            if s == t and first == len(rows) and (first % p == 0
                                                  or self.refs[self.table[s][kept]] == 1):
                kept = -(-first // p)
            new = self.lowest(-(-len(rows) // p) - kept, taken)
            plan.append((s, t, rows, kept, new))
        at = [self.places(s, rows[kept * p:]) for s, t, rows, kept, new in plan]
        dst = [[], []]
        for s, t, rows, kept, new in plan:
            dst[0] += [new[i // p] for i in range(len(rows) - kept * p)]
            dst[1] += [i % p for i in range(len(rows) - kept * p)]
        a, b = torch.cat([x[0] for x in at]), torch.cat([x[1] for x in at])
        if len(a):
            x, y = _i64(dst[0]), _i64(dst[1])
            self.k[:, x, :, y] = self.k[:, a, :, b]
            self.v[:, x, :, y] = self.v[:, a, :, b]
        for s, t, rows, kept, new in plan:
            head = self.table[s][:kept]
            if s == t:
                for q in self.table[s][kept:]:
                    self.refs[q] -= 1
            else:
                for q in head:
                    self.refs[q] += 1
            for q in new:
                self.refs[q] += 1
            self.table[t], self.lens[t] = head + new, len(rows)


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def _parents(rng, rows):
    """Trees of drafted tokens: each row's parent among the few before it, -1 for a root."""
    return [int(rng.integers(max(-1, i - 6), i)) for n in rows for i in range(n)]


def _ptr(rows):
    return [0] + np.cumsum(rows).tolist()


def _positions(rng, n, axes):
    """Text and image rows mixed: the axes agree for text, and part for images."""
    at = np.arange(n) + int(rng.integers(0, 100000))
    pos = np.tile(at, (axes, 1))
    image = rng.random(n) < 0.5
    for a in range(1, axes):
        pos[a, image] = rng.integers(0, 1024, int(image.sum()))
    return _i32(pos.tolist())


def prepare(case, seed):
    c, g = case, _gen(seed, 3)
    rng = np.random.default_rng([seed, 1])
    if c["kind"] == "rope":
        n, h, d = c["tokens"], c["hq"] + c["hkv"], c["d"]
        s = {"case": c, "pos": _positions(rng, n, c["axes"])}
        wide = _normal(g, n, (h + c["hkv"] if c["fused"] else h) * d)
        s["x"] = wide[:, :h * d].view(n, h, d) if c["fused"] else wide.view(n, h, d)
        if c["both"]:
            s["g"] = _normal(g, n, h, d)
        if own:
            from paper_2609_00865_amd import mv
            s["rope"] = mv.RopeAxes(c["d"], _axis_map(c["rot"] // 2, c["axes"], c["layout"]), THETA)
        return s
    page = c["page"]
    if c["kind"] == "fork":
        k, n = c["groups"], c["children"]
        lens = [max(1, c["length"] - 7 * i) for i in range(k)]
        book = _Book(seed, lens, k * (n + 1), k * n + 3, c["layers"], c["hkv"], c["d"], page)
        s = {"case": c, "src": [i for i in range(k) for _ in range(n)],
             "dst": list(range(k, k * (n + 1)))}
    elif c["kind"] == "edit":
        k = c["seqs"]
        cut = [_spans(c, seed, i) for i in range(k)]
        lens = [n for n, _ in cut]
        spare = sum(-(-n // page) + 1 for n in lens) + 3
        book = _Book(seed, lens, 2 * k, spare, c["layers"], c["hkv"], c["d"], page)
        s = {"case": c, "src": list(range(k)), "dst": list(range(k, 2 * k)),
             "spans": [x for _, x in cut]}
    else:
        ctx, rows = _sizes(c)
        k, step = len(ctx), c["kind"] == "step"
        spare = sum(-(-(n + page) // page) + 1 for n in rows) * 2 + 3 if step else 3
        lens = ctx if step else [a + b for a, b in zip(ctx, rows)]
        layers = c["layers"] if step else 1
        book = _Book(seed, lens, 2 * k if step else k, spare, layers, c["hkv"], c["d"], page)
        N = sum(rows)
        s = {"case": c, "seqs": rng.permutation(k).tolist()}
        s["ctx"], s["rows"] = [ctx[i] for i in s["seqs"]], [rows[i] for i in s["seqs"]]
        s["parent"] = _parents(rng, s["rows"]) if step or c["tree"] else None
        s["q"] = _normal(g, layers, N, c["hq"], c["d"])
        if step:
            s["kn"], s["vn"] = (_normal(g, layers, N, c["hkv"], c["d"]) for _ in range(2))
            s["pos"] = _positions(rng, N, 3)
            s["spans"] = []   # the rows of each tree that are not on the accepted path
            at = 0
            for n, m in zip(s["ctx"], s["rows"]):
                keep, i = [], int(rng.integers(0, m))
                while i >= 0:
                    keep.append(i)
                    i = s["parent"][at + i]
                at += m
                keep = sorted(keep)
                edges = [-1] + keep + [m]
                s["spans"].append([(n + a + 1, n + b) for a, b in zip(edges, edges[1:])
                                   if b > a + 1])
    if not own:
        s["book"] = book
        if s.get("parent") is not None:
            s["parent_t"] = _i64(s["parent"])
        return s
    from paper_2609_00865_amd import mv
    s["cache"] = book.open()
    for name in ("src", "dst", "seqs"):
        if name in s:
            s[name + "_t"] = _i32(s[name])
    if "spans" in s:
        s["span_ptr"] = _i32(_ptr([len(x) for x in s["spans"]]))
        s["span_t"] = _i32([list(x) for y in s["spans"] for x in y] or [[0, 0]])
    if "rows" in s:
        s["row_ptr"] = _i32(_ptr(s["rows"]))
        s["max_len"] = max(a + b for a, b in zip(s["ctx"], s["rows"]))
        if s["parent"] is not None:
            s["parent_t"] = _i32(s["parent"])
    if c["kind"] == "step":
        s["rope"] = mv.RopeAxes(c["d"], _axis_map(c["d"] // 2, 3, "sections"), THETA)
        s["dst_t"] = _i32([len(s["seqs"]) + i for i in s["seqs"]])
        s["cut_ptr"] = _i32(list(range(len(s["seqs"]) + 1)))
        s["cut_t"] = _i32([[n, INF] for n in s["ctx"]])
    return s


# --------------------------------------------------------------------------
# one pass, in plain torch
# --------------------------------------------------------------------------
def _rotate(x, pos, axis, inverse):
    """x [n, heads, d]: the pairs (i, i + pairs) turned by pos[axis(i)] * theta^(-i / pairs)."""
    n = len(axis)
    freq = THETA ** (-torch.arange(n, dtype=torch.float64, device=DEV) / n)
    a = pos[_i64(axis)].to(torch.float64).t() * freq
    c, s = a.cos().float()[:, None], a.sin().float()[:, None]
    if inverse:
        s = -s
    y = x.float()
    u, w = y[..., :n], y[..., n:2 * n]
    return torch.cat([u * c - w * s, w * c + u * s, y[..., 2 * n:]], -1).to(x.dtype)


def _tree_rows(parent, n):
    """[n, n]: which drafted rows each row sees (itself and its ancestors): the
    step to the parent (a root's to itself), doubled until it spans the tree."""
    at = torch.arange(n, device=DEV)
    see = torch.eye(n, device=DEV)
    see[at, torch.where(parent < 0, at, parent)] = 1.0
    for _ in range((n - 1).bit_length()):
        see = (torch.matmul(see, see) > 0).float()
    return see > 0


def _attend(book, layer, q, seqs, rows, parent):
    """Attention of each sequence's newest rows over its rows in the cache."""
    N, hq, d = q.shape
    hkv = book.k.shape[2]
    g, at, o, lse = hq // hkv, 0, [], []
    for s, n in zip(seqs, rows):
        pages, L = _i64(book.table[s]), book.lens[s]
        k = book.k[layer][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :L].float()
        v = book.v[layer][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :L].float()
        see = torch.ones(n, L, dtype=torch.bool, device=DEV)
        see[:, L - n:] = (_tree_rows(parent[at:at + n], n) if parent is not None
                          else torch.ones(n, n, dtype=torch.bool, device=DEV).tril())
        x = q[at:at + n].float().view(n, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, n * g, d)
        z = torch.matmul(x, k.transpose(1, 2)) * (1.0 / math.sqrt(d))
        z = z.masked_fill(~see.repeat_interleave(g, 0), -math.inf)
        m = z.max(-1, keepdim=True).values
        p = torch.exp(z - m)
        t = p.sum(-1, keepdim=True)
        y = torch.matmul(p, v) / t
        o.append(y.view(hkv, n, g, d).permute(1, 0, 2, 3).reshape(n, hq, d))
        lse.append((m + t.log()).view(hkv, n, g).permute(1, 0, 2).reshape(n, hq))
        at += n
    return torch.cat(o).to(q.dtype), torch.cat(lse).t().contiguous()


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rope":
        axis = _axis_map(c["rot"] // 2, c["axes"], c["layout"])
        y = _rotate(s["x"], s["pos"], axis, False)
        return (y, _rotate(s["g"], s["pos"], axis, True)) if c["both"] else (y,)
    b = s["book"]
    if c["kind"] == "attn":
        return _attend(b, 0, s["q"][0], s["seqs"], s["rows"], s.get("parent_t"))
    if c["kind"] == "fork":
        b.free(s["dst"])
        b.compact(s["src"], s["dst"], [[] for _ in s["src"]])
        return (b.k, b.v) + b.tensors()
    if c["kind"] == "edit":
        b.free(s["dst"])
        if c["in_place"]:
            b.compact(s["src"], s["dst"], [[] for _ in s["src"]])
            b.compact(s["dst"], s["dst"], s["spans"])
        else:
            b.compact(s["src"], s["dst"], s["spans"])
        return (b.k, b.v) + b.tensors()
    seqs, k = s["seqs"], len(s["seqs"])
    dst = [k + i for i in seqs]
    b.free(dst)
    b.compact(seqs, seqs, [[(n, INF)] for n in s["ctx"]])
    slot, _ = b.reserve(seqs, s["rows"])
    pages, places = _i64([x // b.page for x in slot]), _i64([x % b.page for x in slot])
    axis = _axis_map(c["d"] // 2, 3, "sections")
    out = []
    for layer in range(c["layers"]):
        b.k[layer, pages, :, places] = _rotate(s["kn"][layer], s["pos"], axis, False)
        b.v[layer, pages, :, places] = s["vn"][layer]
        q = _rotate(s["q"][layer], s["pos"], axis, False)
        out += [q, *_attend(b, layer, q, seqs, s["rows"], s["parent_t"])]
    b.compact(seqs, dst, s["spans"])
    return tuple(out) + (b.k, b.v) + b.tensors()


# --------------------------------------------------------------------------
# one pass, through the library
# --------------------------------------------------------------------------
def _run_own(s):
    from paper_2609_00865_amd import mv
    c = s["case"]
    if c["kind"] == "rope":
        y = mv.rope_axes(s["x"], s["pos"], s["rope"])
        return (y, mv.rope_axes(s["g"], s["pos"], s["rope"], inverse=True)) if c["both"] else (y,)
    cache = s["cache"]
    if c["kind"] == "attn":
        tree = None
        if c["tree"]:
            tree, _ = mv.tree_mask(s["parent_t"], s["row_ptr"], max(s["rows"]))
        return mv.tree_attn(cache, 0, s["q"][0], s["seqs_t"], s["row_ptr"], tree=tree,
                            max_len=s["max_len"])
    state = (cache.k, cache.v, cache.page_table, cache.seq_len, cache.page_refs)
    if c["kind"] == "fork":
        mv.cache_free(cache, s["dst_t"])
        mv.cache_fork(cache, s["src_t"], s["dst_t"])
        return state
    if c["kind"] == "edit":
        mv.cache_free(cache, s["dst_t"])
        if c["in_place"]:
            mv.cache_fork(cache, s["src_t"], s["dst_t"])
            mv.cache_compact(cache, s["dst_t"], s["dst_t"], s["span_ptr"], s["span_t"])
        else:
            mv.cache_compact(cache, s["src_t"], s["dst_t"], s["span_ptr"], s["span_t"])
        return state
    seqs, dst, ptr = s["seqs_t"], s["dst_t"], s["row_ptr"]
    mv.cache_free(cache, dst)
    mv.cache_compact(cache, seqs, seqs, s["cut_ptr"], s["cut_t"])
    slot, _ = mv.cache_reserve(cache, seqs, ptr, s["kn"].shape[1])
    tree, _ = mv.tree_mask(s["parent_t"], ptr, max(s["rows"]))
    out = []
    for layer in range(c["layers"]):
        mv.cache_write(cache, layer, slot, s["kn"][layer], s["vn"][layer], rope=s["rope"],
                       pos=s["pos"])
        q = mv.rope_axes(s["q"][layer], s["pos"], s["rope"])
        out += [q, *mv.tree_attn(cache, layer, q, seqs, ptr, tree=tree, max_len=s["max_len"])]
    mv.cache_compact(cache, seqs, dst, s["span_ptr"], s["span_t"])
    return tuple(out) + state


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "rope":
        n, h, twice = c["tokens"], c["hq"] + c["hkv"], 2 if c["both"] else 1
        return {"bytes": twice * (2 * n * h * c["d"] * 2 + 4 * n * c["axes"]),
                "flops": twice * 3 * n * h * c["rot"]}
    row = 2 * c["hkv"] * c["d"] * 2   # K and V of one token in one layer
    page = c["page"]
    if c["kind"] == "fork":
        moved = table = 0
        for i in range(c["groups"]):
            n = max(1, c["length"] - 7 * i)
            moved += c["children"] * (n % page)
            table += c["children"] * -(-n // page)
        # the table's entries read and written, and the pages' counts
        return {"bytes": 2 * moved * row * c["layers"] + 24 * table, "flops": 0}
    if c["kind"] == "edit":
        moved = table = 0
        for i in range(c["seqs"]):
            n, cut = _spans(c, 1, i)
            left = n - sum(b - a for a, b in cut)
            moved += left - cut[0][0] // page * page
            if c["in_place"]:
                moved += n % page
            table += -(-n // page)
        return {"bytes": 2 * moved * row * c["layers"] + 24 * table, "flops": 0}
    ctx, rows = _sizes(c)
    hq, d, N = c["hq"], c["d"], sum(rows)
    pairs = sum(a * n + n * (n + 1) // 2 for a, n in zip(ctx, rows))
    attn = {"bytes": sum(a + n for a, n in zip(ctx, rows)) * row + N * hq * (4 * d + 4),
            "flops": 4 * d * hq * pairs}
    if c["kind"] == "attn":
        return attn
    moved = sum(n // 2 + a % page for a, n in zip(ctx, rows))
    per = attn["bytes"] + 2 * N * row + N * hq * d * 4 + 2 * moved * row
    return {"bytes": c["layers"] * per, "flops": c["layers"] * attn["flops"]}


# --------------------------------------------------------------------------
# the same results in 64 bits
# --------------------------------------------------------------------------
F64 = torch.float64


def _turn(x, pos, c, inverse):
    """Rotation as a product of complex numbers, in 64 bits."""
    h = (c["rot"] if "rot" in c else c["d"]) // 2
    layout, axes = (c["layout"], c["axes"]) if "layout" in c else ("sections", 3)
    axis = _i64(_axis_map(h, axes, layout))
    i = torch.arange(h, device=DEV, dtype=F64)
    angle = pos.to(F64).index_select(0, axis) * torch.exp(-(i / h) * math.log(THETA))[:, None]
    w = torch.polar(torch.ones_like(angle), -angle if inverse else angle).t()[:, None]
    y = x.to(F64).clone()
    z = torch.complex(y[..., :h].contiguous(), y[..., h:2 * h].contiguous()) * w
    y[..., :h], y[..., h:2 * h] = z.real, z.imag
    return y


def _visible(n, L, parent):
    """[n, L] on the host: context rows, and among the newest n a row's ancestors or predecessors."""
    m = np.ones((n, L), dtype=bool)
    for i in range(n):
        if parent is None:
            m[i, L - n + i + 1:] = False
        else:
            m[i, L - n:] = False
            j = i
            while j >= 0:
                m[i, L - n + j] = True
                j = int(parent[j])
    return torch.from_numpy(m).to(DEV)


def _attend64(k, v, q, see):
    """k, v [L, hkv, d], q [n, hq, d] (64 bits): one query head at a time."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    o, lse = torch.empty_like(q), torch.empty(hq, n, dtype=F64, device=DEV)
    for h in range(hq):
        z = (q[:, h] @ k[:, h // g].t()) / math.sqrt(d)
        z[~see] = -math.inf
        lse[h] = torch.logsumexp(z, 1)
        o[:, h] = torch.exp(z - lse[h][:, None]) @ v[:, h // g]
    return o, lse


def _all_attend64(pool_k, pool_v, b, lens, table, q, seqs, rows, parent):
    o, lse, at = [], [], 0
    for s, n in zip(seqs, rows):
        L = lens[s]
        r = np.arange(L)
        page, place = _i64(np.asarray(table[s])[r // b.page].tolist()), _i64((r % b.page).tolist())
        k, v = pool_k[page, :, place].to(F64), pool_v[page, :, place].to(F64)
        par = parent[at:at + n] if parent is not None else None
        a, z = _attend64(k, v, q[at:at + n].to(F64), _visible(n, L, par))
        o.append(a)
        lse.append(z)
        at += n
    return torch.cat(o), torch.cat(lse, 1)


def _branch64(pools, page, table, refs, n, cut, held):
    """Pools after a copy of sequence `table` (n rows) without the rows of
    `cut` is laid down behind its whole pages before the first of them; its new table."""
    live = np.ones(n, dtype=bool)
    for a, b in cut:
        live[a:b] = False
    rows = np.flatnonzero(live)
    first = int(np.argmin(live)) if not live.all() else n
    keep = first // page
    empty = [i for i in range(len(refs)) if refs[i] == 0 and i not in held]
    moved = rows[keep * page:]
    new = empty[:-(-len(moved) // page)]
    held.update(new)
    if len(moved):
        src, old = np.asarray(table)[moved // page], moved % page
        i = np.arange(len(moved))
        dst = np.asarray(new)[i // page]
        for pool in pools:
            rows_of = pool[:, _i64(src.tolist()), :, _i64(old.tolist())].clone()
            pool[:, _i64(dst.tolist()), :, _i64((i % page).tolist())] = rows_of
    return list(table[:keep]) + new


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    if c["kind"] == "rope":
        y = _turn(s["x"], s["pos"], c, False)
        return (y, _turn(s["g"], s["pos"], c, True)) if c["both"] else (y,)
    b = s["book"]
    if c["kind"] == "attn":
        if sum(s["rows"]) * max(b.lens) * c["hq"] * c["d"] > 1 << 41:
            return None
        return _all_attend64(b.k[0], b.v[0], b, b.lens, b.table, s["q"][0], s["seqs"], s["rows"],
                             s["parent"])
    table, lens, refs = [list(t) for t in b.table], list(b.lens), list(b.refs)
    none = (None, None, None)   # page numbers and counts: whole numbers, compared as they are
    if c["kind"] in ("fork", "edit"):
        pools = [b.k, b.v]
        held, after = set(), {}
        if c["kind"] == "fork" or c["in_place"]:
            for x, y in zip(s["src"], s["dst"]):
                after[y] = _branch64(pools, b.page, table[x], refs, lens[x], [], held)
        if c["kind"] == "edit":
            base = after if c["in_place"] else dict(zip(s["dst"], (table[x] for x in s["src"])))
            held2 = set(held)
            for x, y, cut in zip(s["src"], s["dst"], s["spans"]):
                _branch64(pools, b.page, base[y], refs, lens[x], cut, held2)
        return tuple(p.to(F64) for p in pools) + none
    # a verification step: rows reserved, rotated and written, attended, the path kept
    page, held, place = b.page, set(), []
    empty = [i for i in range(len(refs)) if refs[i] == 0]
    for q, n in zip(s["seqs"], s["rows"]):
        for r in range(lens[q], lens[q] + n):
            if r // page == len(table[q]):
                table[q].append(empty.pop(0))
                held.add(table[q][-1])
            place.append((table[q][r // page], r % page))
        lens[q] += n
    x, y = _i64([p for p, _ in place]), _i64([r for _, r in place])
    pk, pv = b.k.to(F64), b.v.to(F64)
    out = []
    for layer in range(c["layers"]):
        kn = _turn(s["kn"][layer], s["pos"], c, False)
        pk[layer, x, :, y] = kn
        pv[layer, x, :, y] = s["vn"][layer].to(F64)
        qn = _turn(s["q"][layer], s["pos"], c, False)
        # attention takes what is stored: q and the cache in their 16 bits
        out += [qn, *_all_attend64(pk[layer].to(torch.bfloat16), pv[layer], b, lens, table,
                                   qn.to(torch.bfloat16), s["seqs"], s["rows"], s["parent"])]
    for q, cut in zip(s["seqs"], s["spans"]):
        _branch64([pk, pv], page, table[q], refs, lens[q], cut, held)
    return tuple(out) + (pk, pv) + none
