"""The cache's operators as they are used together: a record replayed through
the cache against the masked attention of the same record; a group of samples
verified by drafted trees; both as captured graphs, replayed."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as OC
from paper_2609_00865_amd import mv, synth
from tests.parity import assert_bf16_close

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def i32(x, shape=None):
    t = torch.tensor(x, dtype=torch.int32, device="cuda")
    return t if shape is None else t.reshape(shape)


@pytest.mark.parametrize("d,hq,hkv,page", [(128, 14, 2, 16), (64, 4, 4, 64)])
def test_replayed_record_is_the_masked_attention(d, hq, hkv, page):
    """Three trajectories side by side: rows enter in chunks, every edit
    compacts its cache (on half of them into a fork that goes on), and each
    row's attention is mv_attn_fwd's under the view mask of the record."""
    rng = np.random.default_rng(d)
    trajs = synth.random_trajectories(rng, [700, 411, 97], max_edits=5, max_span=60)
    T = trajs[-1].end
    gen = torch.Generator().manual_seed(1)
    q = torch.randn(T, hq, d, generator=gen).to(BF).cuda()
    k, v = (torch.randn(T, hkv, d, generator=gen).to(BF).cuda() for _ in range(2))
    ref_o, ref_lse = mv.attn_fwd(mv.ViewMask(trajs).upload(), q, k, v)
    c = mv.PagedCache(1, 4 * T // page + 20, page, hkv, d, 2 * len(trajs), 700 // page + 2)
    c.k.fill_(float("nan"))      # rows that nobody wrote must not show
    c.v.fill_(float("nan"))
    seq = list(range(len(trajs)))
    live = [[] for _ in trajs]
    at = [t.begin for t in trajs]
    done = [0] * len(trajs)      # edits applied
    o, lse = torch.zeros_like(q), torch.zeros(hq, T, device="cuda")
    while any(a < t.end for a, t in zip(at, trajs)):
        # edits that fire at the next row
        for i, t in enumerate(trajs):
            while done[i] < len(t.edits) and t.edits[done[i]].junction == at[i]:
                gone = {r for a, b in t.edits[done[i]].evict for r in range(a, b)}
                spans = [[j, j + 1] for j, r in enumerate(live[i]) if r in gone]
                to = seq[i] if done[i] % 2 else (seq[i] + len(trajs)) % (2 * len(trajs))
                mv.cache_compact(c, i32([seq[i]]), i32([to]), i32([0, len(spans)]),
                                 i32(spans, (len(spans), 2)))
                if to != seq[i]:
                    mv.cache_free(c, i32([seq[i]]))
                    seq[i] = to
                live[i] = [r for r in live[i] if r not in gone]
                done[i] += 1
        rows, n = [], []
        for i, t in enumerate(trajs):
            end = min([t.end, at[i] + int(rng.integers(1, 80))] +
                      [e.junction for e in t.edits[done[i]:done[i] + 1]])
            rows += range(at[i], end)
            live[i] += range(at[i], end)
            n.append(end - at[i])
            at[i] = end
        pick = torch.tensor(rows, device="cuda")
        ids, ptr = i32(seq), i32([0] + np.cumsum(n).tolist())
        slot, _ = mv.cache_reserve(c, ids, ptr, len(rows))
        mv.cache_write(c, 0, slot, k[pick], v[pick])
        o[pick], l = mv.tree_attn(c, 0, q[pick], ids, ptr)
        lse[:, pick] = l
    st = c.status()
    assert st["refused_pages"] == 0 and st["refused_entries"] == 0
    assert c.seq_len[i32(seq).long()].tolist() == [len(x) for x in live]
    assert_bf16_close(o, ref_o, f"replayed record d={d}")
    assert float((lse - ref_lse).abs().max()) < 1e-3
    mv.cache_free(c, i32(seq))
    assert c.status()["free_pages"] == c.shape.n_pages


class Draft:
    """A prompt forked into samples; each verifies a tree and keeps one path."""

    def __init__(self, seed=0, hq=8, hkv=2, d=64, page=16, layers=2):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=gen).to(BF)
        self.hq, self.hkv, self.d, self.page, self.layers = hq, hkv, d, page, layers
        self.prompt, self.samples = 53, 5
        self.n = [7, 12, 1, 9, 20]
        N = sum(self.n)
        self.par = [[int(rng.integers(max(-1, i - 4), i)) for i in range(n)] for n in self.n]
        self.pk, self.pv = r(layers, self.prompt, hkv, d), r(layers, self.prompt, hkv, d)
        self.k, self.v, self.q = r(layers, N, hkv, d), r(layers, N, hkv, d), r(layers, N, hq, d)
        self.pos = torch.randint(0, 4000, (3, N), generator=gen).to(torch.int32)
        self.axis = [i % 3 for i in range(d // 2)]
        self.keep = []
        for p in self.par:
            i, path = len(p) - 1, []
            while i >= 0:
                path.append(i)
                i = p[i]
            self.keep.append(path[::-1])
        self.c = mv.PagedCache(layers, 60, page, hkv, d, 1 + 2 * self.samples, 8)
        self.m = OC.Cache(layers, 60, page, hkv, d, 1 + 2 * self.samples, 8)
        self.c.k.zero_()
        self.c.v.zero_()
        slot, _ = mv.cache_reserve(self.c, i32([0]), i32([0, self.prompt]), self.prompt)
        self.m.reserve([0], [0, self.prompt], self.prompt)
        for x in range(layers):
            mv.cache_write(self.c, x, slot, self.pk[x].cuda(), self.pv[x].cuda())
            self.m.write(x, slot.tolist(), self.pk[x].double().numpy(), self.pv[x].double().numpy())
        S = self.samples
        self.ids, self.out_ids = list(range(1, 1 + S)), list(range(1 + S, 1 + 2 * S))
        self.spans = []
        for p, path in zip(self.par, self.keep):
            edges = [-1] + path + [len(p)]
            self.spans.append([[self.prompt + a + 1, self.prompt + b]
                               for a, b in zip(edges, edges[1:]) if b > a + 1])
        self.dev = {n: getattr(self, n).cuda() for n in ("k", "v", "q", "pos")}
        self.idx = {"src": i32([0] * S), "ids": i32(self.ids), "out": i32(self.out_ids),
                    "all": i32(self.ids + self.out_ids),
                    "ptr": i32([0] + np.cumsum(self.n).tolist()),
                    "par": i32([x for p in self.par for x in p]),
                    "sptr": i32([0] + np.cumsum([len(s) for s in self.spans]).tolist()),
                    "spans": i32([x for s in self.spans for x in s], (-1, 2))}
        self.rope = mv.RopeAxes(d, self.axis, 1e4)

    def step(self):
        """One pass, from the prompt alone to the accepted paths."""
        x, c, out = self.idx, self.c, []
        mv.cache_free(c, x["all"])
        mv.cache_fork(c, x["src"], x["ids"])
        slot, _ = mv.cache_reserve(c, x["ids"], x["ptr"], sum(self.n))
        tree, _ = mv.tree_mask(x["par"], x["ptr"], max(self.n))
        for layer in range(self.layers):
            mv.cache_write(c, layer, slot, self.dev["k"][layer], self.dev["v"][layer],
                           rope=self.rope, pos=self.dev["pos"])
            q = mv.rope_axes(self.dev["q"][layer], self.dev["pos"], self.rope)
            out += mv.tree_attn(c, layer, q, x["ids"], x["ptr"], tree=tree)
        mv.cache_compact(c, x["ids"], x["out"], x["sptr"], x["spans"])
        return out

    def check(self, out):
        m, S = self.m, self.samples
        m.free(self.ids + self.out_ids)
        m.fork([0] * S, self.ids)
        slot, _ = m.reserve(self.ids, [0] + np.cumsum(self.n).tolist(), sum(self.n))
        rot = lambda x: torch.from_numpy(OC.rotate(x.double().numpy(), self.pos.numpy(), self.axis,
                                                   1e4)).to(BF).double().numpy()
        for layer in range(self.layers):
            m.write(layer, slot, rot(self.k[layer]), self.v[layer].double().numpy())
            q, at = rot(self.q[layer]), 0
            for s, p in zip(self.ids, self.par):
                n = len(p)
                k, v = m.gather(layer, s)
                see = np.ones((n, len(k)), dtype=bool)
                see[:, len(k) - n:] = OC.tree_rows(p, n)[0]
                o, lse, _ = OC.attend(k, v, q[at:at + n], see, 1 / math.sqrt(self.d))
                assert_bf16_close(out[2 * layer][at:at + n], torch.from_numpy(o), "drafted rows")
                # a rotated key may round to the other neighbour: half an ulp of K moves a score
                assert np.abs(out[2 * layer + 1][:, at:at + n].double().cpu().numpy() - lse).max() < 2e-2
                at += n
        m.compact(self.ids, self.out_ids, self.spans)
        assert self.c.seq_len.tolist() == m.len
        assert self.c.page_refs.tolist() == m.refs
        assert np.array_equal(self.c.page_table.cpu().numpy(), m.page_table())
        assert self.c.seq_len[self.idx["out"].long()].tolist() == [self.prompt + len(p)
                                                                  for p in self.keep]
        for dev, ref in ((self.c.k, m.k), (self.c.v, m.v)):
            x = dev.cpu().double().numpy()
            assert (np.abs(x - ref) <= 2.0 ** -7 * np.abs(ref)).all()   # one ulp: a rounding that fell the other way


@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 2), (128, 7, 1)])
def test_drafted_trees(d, hq, hkv):
    s = Draft(d, hq, hkv, d)
    s.check(s.step())
    s.check(s.step())


def test_captured_steps():
    """Two caches' steps as graphs, replayed in turn with eager work between;
    every replay equals the eager pass."""
    steps = [Draft(1), Draft(2, hq=7, hkv=1, d=128, page=32)]
    eager = [[t.clone() for t in s.step()] for s in steps]
    pools = [(s.c.k.clone(), s.c.v.clone(), s.c.page_table.clone(), s.c.page_refs.clone()) for s in steps]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in steps:
        with torch.cuda.stream(side):
            s.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.step())
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1, 0):
            for t in outs[i]:
                t.fill_(3.0)
            graphs[i].replay()
            if turn % 2:
                torch.cuda.synchronize()
                steps[1 - i].step()
            torch.cuda.synchronize()
            for a, b in zip(outs[i], eager[i]):
                assert torch.equal(a, b), (turn, i)
            s = steps[i]
            for a, b in zip((s.c.k, s.c.v, s.c.page_table, s.c.page_refs), pools[i]):
                assert torch.equal(a, b)
        assert steps[0].c.status()["refused_entries"] == 0


def test_shared_workspace():
    """One workspace for calls of different sizes, one after another on a stream."""
    s = Draft(3)
    s.step()
    q, x = s.dev["q"][0], s.idx
    ws = mv.tree_attn_workspace(s.c, q, 5)
    a = mv.tree_attn(s.c, 0, q, x["ids"], x["ptr"])
    b = mv.tree_attn(s.c, 1, q[:1], x["ids"][:1], i32([0, 1]))
    for _ in range(2):
        a2 = mv.tree_attn(s.c, 0, q, x["ids"], x["ptr"], workspace=ws)
        b2 = mv.tree_attn(s.c, 1, q[:1], x["ids"][:1], i32([0, 1]), workspace=ws)
        for p, r in zip(a + b, a2 + b2):
            assert torch.equal(p, r)
