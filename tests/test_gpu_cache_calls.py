"""The paged cache's calls from Python: what they share between threads and graphs, and what a refused call leaves behind."""
import threading

import numpy as np
import pytest
import torch

from paper_2406_11209_amd import api
from paper_2406_11209_amd.cache import PagedCache
from test_gpu_cache import check_attend, deal, filled, starts_of

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def attending(seed, length=300):
    cache = filled(PagedCache(128, 2, 40, 16), seed)
    tables, table, lengths = deal(cache, [length, 200], seed + 1)
    return cache, tables, table, lengths


def test_many_short_sequences_without_a_bound_of_their_runs():
    """max_new is an expectation: where none is given, all tokens, and more workgroups than a launch can have must not follow from it."""
    seqs, page = 20000, 16
    cache = filled(PagedCache(32, 2, 64, page, "f16"), 241)
    rng = np.random.default_rng(242)
    pages = rng.integers(0, 64, seqs)
    lengths = rng.integers(1, page + 1, seqs)
    table = torch.from_numpy(pages[:, None].astype(np.int32)).cuda()
    length_t = torch.from_numpy(lengths.astype(np.int32)).cuda()
    q = torch.randn(seqs, 8, 32, device="cuda").to(torch.bfloat16)
    starts = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, float("nan"))
    cache.attend(q, table, length_t, starts=starts, out=out)
    assert bool(torch.isfinite(out.float()).all())
    for first in (0, 6560, 13000, seqs - 40):
        some = slice(first, first + 40)
        check_attend(cache, q[some], out[some], None, [[int(p)] for p in pages[some]], lengths[some].tolist(), [1] * 40)
