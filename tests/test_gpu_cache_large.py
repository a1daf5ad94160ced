"""States taken over by a cache that has been in use, against the plain model."""
import pytest

from tests.test_gpu_cache import Pair, i32

pytestmark = pytest.mark.gpu


def table_of(p):
    return i32(p.m.page_table().tolist()), i32(p.m.len), i32(p.m.refs)


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
