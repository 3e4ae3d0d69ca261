"""The paged cache's limits: what a launch cannot hold is refused before any device work.  No GPU."""
import ctypes

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
