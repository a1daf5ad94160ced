"""The page operators at the sizes that take their planning blocks several
rounds: more entries than threads (1024), searches for free pages past one
round of holders (4096), sequences of many pages.  Against the plain model, as
the small calls are: tables, lengths, holders, counts and pools bit for bit."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache import Pair, i32

pytestmark = pytest.mark.gpu


def table_of(p):
    return i32(p.m.page_table().tolist()), i32(p.m.len), i32(p.m.refs)


def ptr_of(rows):
    return [0] + np.cumsum(rows).tolist()


def spans_of(rng, n, top):
    cut = []
    for _ in range(n):
        at = np.sort(rng.choice(top, size=2 * int(rng.integers(0, 4)), replace=False))
        cut.append([(int(a), int(b)) for a, b in zip(at[::2], at[1::2])])
    return cut


def test_more_entries_than_threads():
    """2600 entries a call, with repeats, padding and bad ids on both sides of
    the 1024th: reserved, made longer (some past their table), forked, edited
    in place and into branches, freed."""
    rng = np.random.default_rng(3)
    p = Pair(layers=1, pages=7000, heads=1, seqs=2700, max_pages=4, seed=2)
    ids = rng.permutation(2500).tolist()
    for at, x in ((7, -1), (900, 2700), (1023, ids[3]), (1024, ids[1024]), (1500, ids[2]),
                  (1501, -1), (2049, -9), (2300, ids[1200]), (2301, ids[2000])):
        ids.insert(at, x)
    rows = rng.integers(0, 50, len(ids)).tolist()
    print("[gpu] reserve, 2509 entries", flush=True)
    p.reserve(ids, ptr_of(rows))
    p.status()
    p.reserve(ids[::-1], ptr_of(rng.integers(0, 30, len(ids)).tolist()))
    p.status()
    gone = ids[1:2400:2]
    print("[gpu] free, 1200 entries", flush=True)
    p.free(gone)
    p.status()
    held, empty = [s for s in range(2700) if p.m.len[s]], [s for s in range(2700) if not p.m.len[s]]
    dst = rng.permutation(empty).tolist()[:1300]
    src = [held[i % len(held)] for i in range(1300)]
    for at in (5, 1030, 1299):
        dst[at] = dst[0]                          # a target named before
    dst[1100], src[1200] = held[0], 2700          # a full target, a bad source
    print("[gpu] fork, 1300 entries", flush=True)
    p.fork(src, dst)
    p.status()
    live = [s for s in range(2700) if p.m.len[s]]
    order = rng.permutation(live).tolist()
    cut = spans_of(rng, len(order), 70)
    cut[4] = [(5, 3)]                             # not sorted
    cut[1400 % len(order)] = [(9, 12), (11, 14)]  # overlapping
    print(f"[gpu] compact, {len(order)} entries", flush=True)
    p.compact(order, order, cut)
    p.status()
    empty = [s for s in range(2700) if not p.m.len[s]]
    n = min(len(empty), len(order), 1200)
    p.compact(order[:n], empty[:n], spans_of(rng, n, 40))
    p.status()
    again = rng.permutation(2700).tolist()
    again[2000:2000] = again[:3] + [-1, 2700] + again[1500:1502]
    print("[gpu] free, 2707 entries", flush=True)
    p.free(again)
    assert p.m.free_pages() == 7000
    p.status()


@pytest.mark.parametrize("first", [1100, 900])
def test_pages_run_out_among_many_entries(first):
    """The entry that some of its pages were dealt to lies behind (before) the
    1024th; what was dealt to it is free again, entries that need none go on."""
    p = Pair(layers=1, pages=2000, heads=1, seqs=2600, max_pages=4, seed=1)
    rows = [16] * first + [40] * 500 + [0, 5] * 20
    p.reserve(list(range(len(rows))), ptr_of(rows))
    p.status()
    p.free(list(range(0, first, 2)))
    p.reserve(list(range(1700, 1900)), ptr_of([33] * 200))       # dealt from the first free ones on
    p.status()
    live = [s for s in range(2600) if p.m.len[s]]
    empty = [s for s in range(2600) if not p.m.len[s]]
    n = min(len(live), len(empty))
    print(f"[gpu] copies, {n} entries", flush=True)
    p.fork(live[:n], empty[:n], share=False)
    p.status()
    p.free(list(range(2600)))
    p.status()


def test_search_past_one_round():
    """Free pages behind thousands of held ones, in one run and in several,
    enough of them and not; a low one freed before a search that ends high."""
    p = Pair(layers=1, pages=10241, heads=1, seqs=6, max_pages=6000, seed=4)
    print("[gpu] search", flush=True)
    p.reserve([5], [0, 33])                                      # the first three
    p.reserve([0], [0, 5000 * 16])
    p.reserve([1], [0, 4300 * 16 - 3])                           # rounds 2 and 3
    p.free([5])
    p.reserve([2, 5], [0, 1500 * 16, 1500 * 16 + 5])             # 3 + 938 free: rolled back
    p.status()
    p.reserve([5], [0, 33])                                      # the first three again
    p.fork([1, 0], [2, 3])                                       # one part-filled page
    p.status()
    p.free([0, 3])                                               # 5000 low ones free
    p.reserve([4], [0, 5300 * 16])                               # across the held ones
    p.status()
    p.free([5])
    p.fork([4, 1], [0, 5], share=False)                          # first and last round: rolled back
    p.status()
    p.compact([4, 1], [4, 2], [[(5000, 5008), (70000, 80000)], []])   # too few; a full target
    p.reserve([3], [0, 200 * 16])                                # the first three and 197 behind
    p.compact([4], [4], [[(81000, 2 ** 31 - 1)]])                # cut off at the end
    p.free([1])
    p.compact([4], [4], [[(100, 108), (70000, 80000)]])
    p.status()
    p.free([0, 1, 2, 3, 4, 5])
    assert p.m.free_pages() == 10241
    p.status()


def test_a_restored_state_is_searched_from_the_first_page():
    """A state whose free pages lie below where the search had come to."""
    p = Pair(layers=1, pages=60, heads=1, seqs=6, max_pages=40, seed=5)
    p.reserve([0, 1, 2], [0, 20 * 16, 40 * 16, 55 * 16])
    before = table_of(p)
    p.free([0])
    p.reserve([3], [0, 18 * 16])
    p.m.free([1, 3])                                             # the model alone
    p.c.restore(*table_of(p))
    p.same()
    p.reserve([4, 5], [0, 30 * 16, 45 * 16])                     # all that is free
    p.status()
    assert p.m.free_pages() == 0
    p.c.restore(*before)
    assert p.c.status() == {"free_pages": 5, "refused_pages": 0, "refused_entries": 0}
