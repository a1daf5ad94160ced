"""The plain model of the cache against the definition of the live view: a
record replayed through it (rows appended, each edit compacting, a branch
forked before an edit) gives every row the attention of its live view."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import cache as OC
from oracle import views as OV
from paper_2609_00865_amd import synth


def replay(trajs, q, k, v, page, fork_at=None):
    """Attention of every row, each trajectory through a cache of its own."""
    T, hq, d = q.shape
    o, lse = np.zeros((T, hq, d)), np.zeros((hq, T))
    for t in trajs:
        n = t.end - t.begin
        c = OC.Cache(1, 4 * (-(-n // page) + 2), page, k.shape[1], d, 3, -(-n // page) + 1)
        live, s = [], 0
        cuts = [t.begin] + [e.junction for e in t.edits] + [t.end]
        for j, (a, b) in enumerate(zip(cuts, cuts[1:])):
            if j:
                gone = {r for x, y in t.edits[j - 1].evict for r in range(x, y)}
                spans = [(i, i + 1) for i, r in enumerate(live) if r in gone]
                c.compact([s], [s], [spans])
                live = [r for r in live if r not in gone]
            for r in range(a, b):
                slot, pos = c.reserve([s], [0, 1], 1)
                assert pos == [len(live)]
                c.write(0, slot, k[r:r + 1], v[r:r + 1])
                live.append(r)
            kk, vv = c.gather(0, s)
            see = np.ones((b - a, len(live)), dtype=bool)
            see[:, len(live) - (b - a):] = np.tril(np.ones((b - a, b - a), dtype=bool))
            o[a:b], lse[:, a:b], _ = OC.attend(kk, vv, q[a:b], see, 1 / math.sqrt(d))
            if j == fork_at:
                c.fork([s], [2 - s])
                c.free([s])
                s = 2 - s
        c.free([s])
        assert c.free_pages() == c.n_pages and not c.bad and not c.no_pages
    return o, lse


@pytest.mark.parametrize("seed", range(4))
def test_replay_is_the_live_view(seed):
    rng = np.random.default_rng(seed)
    trajs = synth.random_trajectories(rng, [60, 33], max_edits=4, max_span=9)
    T = trajs[-1].end
    q = rng.standard_normal((T, 4, 16))
    k, v = rng.standard_normal((2, T, 2, 16))
    ref = OA.logittree(trajs, *(torch.from_numpy(x) for x in (q, k, v)))
    for page, fork_at in ((16, None), (8, 0)):
        o, lse = replay(trajs, q, k, v, page, fork_at)
        assert np.abs(o - ref[0].numpy()).max() < 1e-12
        assert np.abs(lse - ref[1].numpy()).max() < 1e-12


def test_model_rules():
    c = OC.Cache(1, 5, 16, 1, 4, 4, 3)
    slot, pos = c.reserve([2, 0], [0, 17, 20], 20)
    assert slot[:17] == list(range(17)) and slot[17:] == [32, 33, 34] and pos[17:] == [0, 1, 2]
    c.fork([2], [1])
    assert c.table[1] == [0, 3] and c.refs == [2, 1, 1, 1, 0]
    c.compact([1], [1], [[(0, 3)]])              # a shared page is left to the other
    assert c.no_pages == 0 and c.table[1] == [4] and c.refs == [1, 1, 1, 0, 1]
    c.compact([2], [2], [[(5, 99)]])             # cut off at the end: nothing moves
    assert c.table[2] == [0] and c.len[2] == 5 and c.free_pages() == 2
    assert c.reserve([3], [0, 33], 33)[0] == [-1] * 33 and c.no_pages == 1
    see, depth = OC.tree_rows([-1, 0, 0, 2, 4], 5)
    assert depth == [0, 1, 1, 2, 0] and see[3].tolist() == [True, False, True, True, False]


def test_rotation_by_hand():
    x = np.array([[[1.0, 0.0, 0.0, 2.0, 7.0]]])
    y = OC.rotate(x, [[1], [3]], [0, 1], 4.0)
    assert np.allclose(y[0, 0], [math.cos(1), -2 * math.sin(1.5), math.sin(1), 2 * math.cos(1.5), 7])
    assert np.allclose(OC.rotate(y, [[1], [3]], [0, 1], 4.0, inverse=True), x)
