"""The paged cache's limits: what a launch cannot hold is refused before any device work.  No GPU."""
import ctypes

import numpy as np
import pytest

from paper_2406_11209_amd import api, cache
from paper_2406_11209_amd.api import Codec
from test_cache_host import FAKE, attention, geometry


def test_more_workgroups_than_a_launch_counts():
    """HIP counts a dimension's threads modulo 2^32 and leaves the others out without an error: 2^24 workgroups of 256."""
    lib, need = cache._library(), ctypes.c_size_t()
    wide, narrow = Codec((256,)), Codec((32,))

    def workspace(codec, g, **changes):
        return lib.pbz_cache_attend_workspace(codec._h, g, attention(**changes), need)

    x = cache._Lines(FAKE, 0, 0)
    assert lib.pbz_cache_append(wide._h, geometry(), 1 << 26, x, x, api.PBZ_BF16, FAKE, None) == -7
    assert lib.pbz_cache_append(narrow._h, geometry(heads=1), 1 << 30, x, x, api.PBZ_BF16, FAKE, None) == -7
    # queries: 16 rows of 256 to a workgroup
    assert workspace(wide, geometry(heads=1), q_heads=1, n_tokens=(1 << 28) - 16, max_new=1) == 0
    assert workspace(wide, geometry(heads=1), q_heads=1, n_tokens=1 << 28, max_new=1) == -7
    # a workgroup for every head of every sequence
    single = dict(starts=None, q_heads=2, max_pages=1, table_stride=1)
    assert workspace(narrow, geometry(), n_tokens=(1 << 23) - 1, n_seqs=(1 << 23) - 1, **single) == 0
    assert workspace(narrow, geometry(), n_tokens=1 << 23, n_seqs=1 << 23, **single) == -7
    # ... whose row blocks are fewer where an expectation of the new tokens asks for more than there can be
    assert workspace(narrow, geometry(), n_tokens=1 << 20, n_seqs=1 << 20, max_new=1 << 20, max_pages=1, table_stride=1) == 0


def test_pairs_that_int32_would_make_other_pages():
    for pairs in (np.array([[1, 2 ** 32 + 3]]), np.array([[2 ** 32 + 1, 3]], dtype=np.uint64), np.array([[-2 ** 32 + 1, 3]]), [(2 ** 33, 1)],
                  [(2 ** 70, 1)], np.array([[2 ** 63 + 1, 3]], dtype=np.uint64)):
        with pytest.raises(api.PbzError) as e:
            cache._pairs(pairs)
        assert e.value.status == -15
    for pairs in (np.array([[1.5, 3.0]]), [[1, 2, 3, 4, 5, 6]], np.array([[1, 2, 3], [4, 5, 6]]), [1, 2, 3], 7, [("a", "b")], [(None, 1)],
                  np.array([[True, False]])):
        with pytest.raises(ValueError):
            cache._pairs(pairs)
    for pairs, want in (([], []), (np.zeros((0, 2), np.int64), []), ([(3, 1)], [(3, 1)]), (np.array([[5, 6], [7, 8]]).T[::-1].T, [(6, 5), (8, 7)]),
                        (np.array([1, 2, 3, 4], dtype=np.uint8), [(1, 2), (3, 4)]), ([(np.int64(9), 2)], [(9, 2)])):
        got = cache._pairs(pairs)
        assert got.dtype == np.int32 and got.flags.c_contiguous and got.tolist() == [list(p) for p in want]


def test_tables_whose_positions_32_bits_nearly_do_not_count():
    """The kernels look up to 256 positions ahead; past 2^31 that was a place in front of the table."""
    lib, need, codec = cache._library(), ctypes.c_size_t(), Codec((64,))
    for page, most in ((16, (1 << 27) - 64), (1024, (1 << 21) - 1)):
        for pages, status in ((most, 0), (most + 1, -7)):
            a = attention(max_pages=pages, table_stride=pages, n_seqs=1, n_tokens=1, starts=None)
            assert lib.pbz_cache_attend_workspace(codec._h, geometry(page_size=page), a, need) == status
