"""Attention over the cache where a workgroup's run of the deal is many units of
64 keys: the loops over keys of both dealt kernels, pages past the first windows
of their ids, maxima that move along a run, masked tiles behind long contexts,
a tile's own cost in the deal, more tile places and entries than one block of
the deal holds.  Every call asserts what it reaches (``Long.deal``).

Tolerance of o against the plain form in 64 bits, element by element: its
rounding to bf16 (2^-8 |o|, twice the half step of 2^-9), and as a relative
error of the weights (which sum w |v| scales): their rounding to bf16 (2^-8),
the scores' (fp32 sums of d products, e = d 2^-24 sum |q k| scale, on both sides
of the quotient: 2 e), fp32 sums of L terms (L 2^-24), the exponential (2^-20;
its argument's rounding is inside e), and up to one rescaling for every 32 keys,
each an exponential and two roundings (2^-21).  lse: e, the same sums and
rescalings, and its own rounding.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache as OC
from paper_2609_00865_amd import mv

pytestmark = pytest.mark.gpu
BF, F64 = torch.bfloat16, torch.float64


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Long:
    """A cache whose sequences have the given lengths on scattered pages, and q
    of each entry's new rows."""

    def __init__(self, lens, rows, hq, hkv, d, page=16, seed=0, ids=None, stale=None):
        need = [-(-n // page) for n in lens]
        pages = sum(need) + 3
        order = np.random.default_rng(seed).permutation(pages).tolist()
        self.table = [[order.pop() for _ in range(n)] for n in need]
        self.lens, self.rows, self.page, self.hq, self.hkv, self.d = lens, rows, page, hq, hkv, d
        self.ids = list(range(len(lens))) if ids is None else ids
        wide = max(need + [1]) + 2
        self.c = mv.PagedCache(1, pages, page, hkv, d, len(lens), wide)
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in (self.c.k, self.c.v):
            x.normal_(generator=g)
        self.q = torch.empty(sum(rows), hq, d, dtype=BF, device="cuda").normal_(generator=g)
        refs = torch.zeros(pages, dtype=torch.int32)
        for t in self.table:
            refs[torch.tensor(t, dtype=torch.long)] = 1
        self.c.restore(i32([t + [-1] * (wide - len(t)) for t in self.table]), i32(lens), refs.cuda())
        if stale is not None:      # every row that no sequence holds
            dead = torch.ones(pages, page, dtype=torch.bool, device="cuda")
            for s in range(len(lens)):
                dead[self.at(s)] = False
            for x in (self.c.k, self.c.v):
                x[0].transpose(1, 2)[dead] = stale
        self.ptr = [0] + np.cumsum(rows).tolist()

    def at(self, s):
        r = np.arange(self.lens[s])
        pages = np.asarray(self.table[s], dtype=np.int64)[r // self.page]
        return torch.from_numpy(pages).cuda(), torch.from_numpy(r % self.page).cuda()

    def of(self, pool, s):
        """Rows of sequence s in 64 bits, [L, hkv, d]."""
        p, r = self.at(s)
        return pool[0, p, :, r].to(F64)

    def put(self, pool, s, r, h, e, x):
        pool[0, self.table[s][r // self.page], h, r % self.page, e] = x

    def deal(self, tree=None, max_len=0):
        """(many pairs, units of a run, what a tile counts for, tile places), by
        the library's rule for calls that are dealt."""
        G, B = self.hq // self.hkv, len(self.rows)
        many = sum(self.rows) * G > 32 * B
        R = 128 if many else 32
        places = sum(self.rows) * G // R + B
        groups = 512 if max_len <= 0 else min(512, places * self.hkv * (-(-max_len // 64)))
        units = tiles = 0
        for s, n in zip(self.ids, self.rows):
            L = self.lens[s] if 0 <= s < len(self.lens) else 0
            for m0 in range(0, n * G, R):
                last = (min(m0 + R, n * G) - 1) // G
                k = L if tree is not None else max(0, L - n + last + 1)
                units += max(1, -(-k // 64))
                tiles += 1
        extra = (6 if many else 4) if units * self.hkv >= 8 * groups else 0
        return many, (units + extra * tiles) * self.hkv / groups, extra, places

    def run(self, tree=None, **kw):
        return mv.tree_attn(self.c, 0, self.q, i32(self.ids), i32(self.ptr), tree=tree, **kw)

    def plain(self, b, see):
        """Entry b in 64 bits: o, lse, sum w |v|, and e; see [n, L]."""
        s, n = self.ids[b], self.rows[b]
        k, v = self.of(self.c.k, s), self.of(self.c.v, s)
        q = self.q[self.ptr[b]:self.ptr[b] + n].to(F64)
        scale, G = 1.0 / math.sqrt(self.d), self.hq // self.hkv
        o, mag = torch.zeros_like(q), torch.zeros_like(q)
        lse = torch.zeros(self.hq, n, dtype=F64, device="cuda")
        e = torch.zeros(n, self.hq, dtype=F64, device="cuda")
        empty = ~see.any(1)
        for h in range(self.hq):
            kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
            z = torch.mm(q[:, h].contiguous(), kh.t().contiguous()) * scale
            z.masked_fill_(~see, -math.inf)
            m = z.max(1, keepdim=True).values.masked_fill(empty[:, None], 0.0)
            w = torch.exp(z - m)
            t = w.sum(1, keepdim=True)
            lse[h] = (m + t.log())[:, 0]
            w = (w / t).masked_fill(empty[:, None], 0.0)
            odd = ~torch.isfinite(vh)
            fin = vh.masked_fill(odd, 0.0)
            o[:, h], mag[:, h] = torch.mm(w, fin), torch.mm(w, fin.abs())
            for r, x in odd.nonzero().tolist():       # left out where it is not seen
                o[:, h, x] += torch.where(see[:, r], w[:, r] * vh[r, x], torch.zeros_like(w[:, r]))
            top = kh.abs().masked_fill(~torch.isfinite(kh), 0.0).max(0).values
            e[:, h] = self.d * 2.0 ** -24 * scale * (q[:, h].abs() @ top)
        return o, lse, mag, e

    def check(self, o, lse, new=None, only=None):
        """new(b, n): [n, n] bool of the new rows each row sees (none: the chain)."""
        o, lse = o.to(F64), lse.to(F64)
        for b, (s, n) in enumerate(zip(self.ids, self.rows)):
            if n == 0 or (only is not None and b not in only):
                continue
            r = slice(self.ptr[b], self.ptr[b] + n)
            L = self.lens[s] if 0 <= s < len(self.lens) else 0
            if L == 0:
                assert (o[r] == 0).all() and torch.isneginf(lse[:, r]).all(), b
                continue
            see = torch.ones(n, L, dtype=torch.bool, device="cuda")
            at = torch.ones(n, n, dtype=torch.bool).tril() if new is None else torch.as_tensor(new(b, n))
            see[:, max(0, L - n):] = at.cuda()[:, max(0, n - L):]
            ro, rl, mag, e = self.plain(b, see)
            steps = L * 2.0 ** -24 + (L / 32 + 1) * 2.0 ** -21 + 2.0 ** -20
            bound = 2.0 ** -8 * ro.abs() + 1.01 * (2.0 ** -8 + 2 * e + steps)[..., None] * mag + 1e-30
            nan, fin = torch.isnan(ro), torch.isfinite(ro)
            assert torch.equal(torch.isnan(o[r]), nan), (b, "NaN where the plain form has none, or not")
            assert torch.equal(o[r][~fin & ~nan], ro[~fin & ~nan]), b
            err = (o[r] - ro).abs()[fin] - bound[fin]
            assert err.numel() == 0 or float(err.max()) <= 0, (b, s, float(err.max()))
            lf = torch.isfinite(rl)
            assert torch.equal(torch.isneginf(lse[:, r]), torch.isneginf(rl)), b
            lerr = (lse[:, r] - rl).abs() - (e.t() + steps + 2.0 ** -22 * rl.abs())
            assert not lf.any() or float(lerr[lf].max()) <= 0, (b, s, float(lerr[lf].max()))


def spread(n, lo, hi):
    """n lengths, uneven, the shortest and the longest among them."""
    return [lo + (i * 7919) % (hi - lo + 1) for i in range(n - 1)] + [hi]


def trees(rng, rows):
    """Parents, which new rows each row sees, and the words on the device."""
    par = [[int(rng.integers(max(-1, i - 5), i)) for i in range(n)] for n in rows]
    seen = [torch.from_numpy(OC.tree_rows(p, len(p))[0]) for p in par]
    tree, _ = mv.tree_mask(i32([x for p in par for x in p]), i32([0] + np.cumsum(rows).tolist()),
                           max(rows))
    return seen, tree


MANY = dict(lens=[3040, 129, 2405, 9013, 1000], rows=[40, 129, 300, 13, 64])


@pytest.mark.parametrize("d,hq,hkv,page", [(128, 8, 2, 16), (64, 7, 1, 16), (128, 16, 1, 64),
                                           (64, 12, 3, 256)])
def test_many_pairs(d, hq, hkv, page):
    """Chunks and trees, about one workgroup to a tile: some 35 tiles of keys in a
    run, pages up to the ninth window of a sequence."""
    s = Long(**MANY, hq=hq, hkv=hkv, d=d, page=page, seed=d + hq)
    many, per, extra, _ = s.deal(max_len=1)
    assert many and per > 16 and extra
    print(f"[gpu] many pairs {hq}/{hkv} d={d} page={page}: {per:.0f} units a run", flush=True)
    s.check(*s.run(max_len=1))
    seen, tree = trees(np.random.default_rng(d), s.rows)
    out = s.run(tree, max_len=1)
    s.check(*out, new=lambda b, n: seen[b])
    again = s.run(tree, max_len=1)
    assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1])


@pytest.mark.parametrize("d,hq,hkv,page,seqs,hi", [(64, 7, 1, 16, 64, 9200), (128, 28, 4, 16, 12, 9000),
                                                   (128, 2, 2, 64, 40, 16000), (64, 32, 1, 256, 30, 8000),
                                                   (64, 16, 8, 16, 6, 60000)])
def test_few_pairs(d, hq, hkv, page, seqs, hi):
    """Single tokens over uneven sequences, dealt to all workgroups: a wave's run
    up to 35 tiles of keys, over several windows of pages."""
    s = Long(spread(seqs, 1, hi), [1] * seqs, hq, hkv, d, page, seed=seqs)
    many, per, extra, _ = s.deal()
    assert not many and per > 4
    print(f"[gpu] few pairs {hq}/{hkv} d={d} page={page}: {per:.0f} units a run, a tile "
          f"{extra}", flush=True)
    s.check(*s.run())


def test_more_tile_places_than_a_block():
    """Of many pairs (256 to a block) and of few (128), a tile's cost counted."""
    s = Long([6007, 300], [5000, 9], 16, 2, 64, 32, seed=1)
    many, per, extra, places = s.deal()
    assert many and extra and places > 256
    print("[gpu] a chunk of 5000 rows", flush=True)
    s.check(*s.run())
    s.check(*s.run(max_len=1))
    s = Long(spread(200, 1, 3001), [1] * 200, 14, 2, 64, 16, seed=2)
    many, per, extra, places = s.deal()
    assert not many and extra and places > 128
    print("[gpu] 200 single tokens", flush=True)
    s.check(*s.run())


@pytest.mark.parametrize("many", [True, False])
def test_more_entries_than_are_held_on_chip(many):
    """700 entries: uneven, some of no rows, padded, naming a sequence again or
    longer than it, with a tile's cost and without."""
    rng = np.random.default_rng(many)
    B, seqs = 700, 300
    lens = spread(seqs, 0, 500 if many else 900)
    ids = [int(x) for x in rng.integers(-1, seqs + 1, B)]
    rows = [int(x) for x in (rng.integers(0, 11, B) if many else rng.integers(0, 3, B))]
    s = Long(lens, rows, 16 if many else 4, 2, 64, 16, seed=3, ids=ids)
    got, per, extra, places = s.deal()
    assert got == many and extra and places > 700
    only = set(range(0, B, 7)) | {B - 1}
    print(f"[gpu] {B} entries, many={many}", flush=True)
    s.check(*s.run(), only=only)
    s.check(*s.run(max_len=1), only=only)
    seen, tree = trees(rng, rows)
    s.check(*s.run(tree), new=lambda b, n: seen[b], only=only)


RAMPS = {"rising": lambda r, L: r / L, "falling": lambda r, L: 1 - r / L,
         "jumps": lambda r, L: float(r // 100 % 3 == 1) - 0.5 * float(r // 100 % 7 == 2)}


@pytest.mark.parametrize("ramp", sorted(RAMPS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("many", [True, False])
def test_maxima_that_move_along_a_run(ramp, d, many):
    """Scores that rise by a hundred from the first key to the last (so that within a
    run probabilities against an earlier maximum pass 2^16), fall, or jump."""
    if many:
        s = Long([4500, 2010], [30, 90], 8, 2, d, 16, seed=d)
        kw = dict(max_len=1)
    else:
        s = Long(spread(40, 100, 9000), [1] * 40, 6, 2, d, 16, seed=d)
        kw = {}
    got, per, _, _ = s.deal(**kw)
    assert got == many and per > (16 if many else 6)
    for x, L in enumerate(s.lens):
        p, r = s.at(x)
        up = torch.tensor([RAMPS[ramp](i, L) for i in range(L)], device="cuda") * 25 * math.sqrt(d)
        s.c.k[0, p, :, r, 0] = up[:, None].to(BF)
    s.q[..., 0] = 4.0
    print(f"[gpu] {ramp} scores, many={many} d={d}", flush=True)
    s.check(*s.run(**kw))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("many", [True, False])
def test_values_that_are_not_finite_behind_a_long_context(bad, d, many):
    """In rows that no sequence holds, in drafted rows that some see and some do
    not (K and V), in masked tiles at the end of runs and in the context."""
    rng = np.random.default_rng(5)
    if many:
        s = Long([5016, 2040, 4097, 1003], [16, 40, 33, 3], 16, 2, d, 16, seed=2, stale=bad)
        kw = dict(max_len=1)
    else:
        s = Long([9906, 9010, 9193, 8003], [6, 10, 1, 3], 16, 8, d, 16, seed=2, stale=bad)
        kw = {}
    seen, tree = trees(rng, s.rows)
    got, per, extra, _ = s.deal(tree, **kw)
    assert got == many and per > 8 and extra
    print(f"[gpu] not finite {bad} many={many} d={d}", flush=True)
    o, lse = s.run(tree, **kw)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    s.check(o, lse, new=lambda b, n: seen[b])
    for b, a in ((0, 2), (1, 7), (1, 1), (3, 1)):         # drafted rows
        r = s.lens[b] - s.rows[b] + a
        s.put(s.c.v, b, r, 0, 5, bad)
        if b == 1:
            s.put(s.c.k, b, r, 1, 9, bad)
    s.check(*s.run(tree, **kw), new=lambda b, n: seen[b])
    s.check(*s.run(**kw))
    for b, r in ((0, 1234), (2, 64), (2, s.lens[2] - 40)):   # context rows, seen by all
        s.put(s.c.v, b, r, 1, 3, bad)
    s.check(*s.run(tree, **kw), new=lambda b, n: seen[b])
    s.put(s.c.k, 2, 700, 0, 8, bad)
    if not math.isinf(bad):                               # (+inf and -inf scores: NaN or no weight)
        s.check(*s.run(tree, **kw), new=lambda b, n: seen[b])


def test_rows_that_see_nothing_over_many_tiles():
    """Words without bits over an empty context: 0 and -inf beside rows that see
    one new row of another tile; an entry longer than its sequence."""
    s = Long([700, 500], [700, 640], 4, 1, 64, 16, seed=1)
    words = np.zeros((1340, 22), dtype=np.uint32)
    see = [np.zeros((n, n), dtype=bool) for n in s.rows]
    for b, i, a in ((0, 3, 699), (0, 200, 0), (0, 201, 64), (0, 699, 127), (1, 5, 639), (1, 600, 141)):
        see[b][i, a] = True
    for b, at in ((0, 0), (1, 700)):
        for i, a in zip(*np.nonzero(see[b])):
            words[at + i, a // 32] |= np.uint32(1) << np.uint32(a % 32)
    tree = torch.from_numpy(words.view(np.int32)).cuda()
    many, per, extra, _ = s.deal(tree, max_len=1)
    assert many and per > 8
    print("[gpu] rows that see nothing", flush=True)
    for kw in (dict(max_len=1), {}):
        o, lse = s.run(tree, **kw)
        s.check(o, lse, new=lambda b, n: see[b])
        assert (o[:3] == 0).all() and torch.isneginf(lse[:, :3]).all()
        assert torch.isfinite(lse[:, 3]).all()
