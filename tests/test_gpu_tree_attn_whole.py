"""The attention's short calls: few pairs of sequences known not to be long,
which one launch takes whole.  The cases of the dealt form again with the longest
sequence named, and sizes where the two forms meet."""
import numpy as np
import pytest
import torch

from oracle import cache as OC
from paper_2609_00865_amd import mv
from tests import test_gpu_tree_attn as T
from tests.test_gpu_tree_attn import BF, Setup, i32, parents

pytestmark = pytest.mark.gpu


def joins(call):
    """The call's result, and how many launches joined partial results."""
    torch.cuda.synchronize()
    mv.profile_enable(True)
    out = call()
    torch.cuda.synchronize()
    n = mv.profile_read("tree_combine")[1]
    mv.profile_enable(False)
    return out, n


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (28, 4), (32, 1), (6, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 256])
def test_single_tokens(hq, hkv, d, page):
    lens = [1, 2, 31, 32, 33, 255, 256, 257, 289, 511, 513, 1023, 1025, 1536]
    s = Setup(lens, [1] * len(lens), hq, hkv, d, page, seed=hq + d)
    print(f"[gpu] whole, single tokens {hq}/{hkv} d={d} page={page}", flush=True)
    out, n = joins(lambda: s.run(max_len=1536))
    assert n == 0
    s.check(*out)
    dealt, n = joins(s.run)
    assert n == 1
    s.check(*dealt)


@pytest.mark.parametrize("d", [64, 128])
def test_longer_than_named(d):
    """Sequences past the length that was named: right, over many windows of pages."""
    lens = [9000, 3, 2311, 1100]
    s = Setup(lens, [1] * 4, 4, 2, d, 16, seed=d)
    out, n = joins(lambda: s.run(max_len=100))
    assert n == 0
    s.check(*out)
    s.check(*s.run(max_len=100000))


@pytest.mark.parametrize("rows,ctx", [([1], [40]), ([5, 4], [0, 300]), ([2, 1, 7, 0, 3], [600, 9, 64, 5, 0])])
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (64, 3, 3)])
def test_trees(rows, ctx, d, hq, hkv):
    rng = np.random.default_rng(sum(rows))
    s = Setup([a + b for a, b in zip(ctx, rows)], rows, hq, hkv, d, 16, seed=8)
    par = [parents(rng, n) for n in rows]
    seen = [OC.tree_rows(p, len(p))[0] for p in par]
    tree, _ = mv.tree_mask(i32([x for p in par for x in p]), i32(s.ptr()), max(rows))
    out, n = joins(lambda: s.run(tree, max_len=max(s.lens)))
    assert n == 0
    s.check(*out, see_new=lambda b, n: seen[b])
    s.check(*s.run(max_len=max(s.lens)))


def test_the_dealt_cases(monkeypatch):
    """Rows that see nothing, values that are not finite where they are seen and
    where not, large scores, a layer of several, calls past the last row."""
    run = Setup.run
    monkeypatch.setattr(Setup, "run", lambda self, tree=None, **kw: run(
        self, tree, **{"max_len": max(1, *self.lens), **kw}))
    T.test_rows_that_see_nothing()
    T.test_a_context_that_is_not_finite()
    T.test_large_scores()
    T.test_uneven_batch()
    for d in (64, 128):
        for bad in (float("nan"), float("inf"), -float("inf"), 3e38):
            T.test_unseen_rows_do_not_show(bad, d)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_rows_of_few(bad, d):
    """As there, with so few pairs that tiles are taken whole."""
    rng = np.random.default_rng(12)
    rows, ctx = [6, 10, 1, 3], [50, 0, 31, 30]
    s = Setup([a + b for a, b in zip(ctx, rows)], rows, 6, 2, d, 16, seed=2, stale=bad)
    par = [parents(rng, n) for n in rows]
    seen = [OC.tree_rows(p, len(p))[0] for p in par]
    tree, _ = mv.tree_mask(i32([x for p in par for x in p]), i32(s.ptr()), max(rows))
    for b, a in ((0, 2), (1, 7), (3, 1)):
        r = s.lens[b] - rows[b] + a
        s.v[0, s.table[b][r // 16], 0, r % 16, 5] = bad
    s.dev(s.c.shape.max_pages)
    (o, lse), n = joins(lambda: s.run(tree, max_len=100))
    assert n == 0
    s.check(o, lse, see_new=lambda b, n: seen[b])


@pytest.mark.parametrize("seqs,hkv,longest,whole", [(1, 4, 1536, 1), (1, 4, 1537, 0), (16, 4, 4096, 1),
                                                    (16, 4, 4097, 0), (64, 4, 1536, 1),
                                                    (64, 4, 1537, 0), (120, 4, 1536, 1),
                                                    (128, 4, 1536, 0)])
def test_where_the_forms_meet(seqs, hkv, longest, whole):
    """Either side of each bound of the rule, the same answers."""
    lens = [1 + 7 * i % 40 for i in range(seqs)]
    s = Setup(lens, [1] * seqs, hkv, hkv, 64, 16, seed=seqs)
    out, n = joins(lambda: s.run(max_len=longest))
    assert n == 1 - whole
    s.check(*out)


def test_padded_batch_and_rows_behind():
    """Padded entries give 0 and -inf; rows past the last entry are left as they were."""
    s = Setup([70, 5], [1, 1, 1, 1], 4, 2, 64, 16, seed=4, ids=[1, -1, 0, 99])
    o = torch.full((7, 4, 64), 5.0, dtype=BF, device="cuda")
    lse = torch.full((4, 7), 5.0, device="cuda")
    q = torch.zeros(7, 4, 64, dtype=BF, device="cuda")
    q[:4] = s.q.cuda()
    mv.tree_attn(s.c, 0, q, i32(s.ids), i32(s.ptr()), max_len=70, out=(o, lse))
    assert (o[4:] == 5).all() and (lse[:, 4:] == 5).all()
    s.check(o[:4], lse[:, :4])
