"""Index arrays that may be left out are checked like the others where they are given."""
import ctypes

import pytest

from paper_2609_00865_amd import mv
from tests.test_cache_abi import FAKE, ODD, R, cache, shape, status


@pytest.mark.parametrize("bad", [ODD, ctypes.c_void_p((1 << 20) + 1)])
def test_optional_arrays(bad):
    s, c = shape(), cache()
    assert status(mv.mv_cache_reserve(R(s), R(c), 1, FAKE, FAKE, 2, None, bad, None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_cache_reserve(R(s), R(c), 1, FAKE, FAKE, 2, FAKE, bad, None)) == "MV_ERR_INVALID_ARG"
    assert status(mv.mv_tree_mask(1, 4, FAKE, FAKE, 1, FAKE, bad, None)) == "MV_ERR_INVALID_ARG"
