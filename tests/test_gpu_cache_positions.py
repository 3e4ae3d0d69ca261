"""Attention over the paged cache sees each position once, and no other: results that tell every position apart (position_code.py; that any single
one shows is tested in test_cache_position_code.py)."""
import numpy as np
import pytest
import torch

import position_code as code
from paper_2406_11209_amd.cache import PagedCache
from test_gpu_cache import check_attend, deal, filled, matrix, starts_of

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def coded(case):
    dim, heads, groups, page, lengths, new, causal, window, holes = case
    cache = PagedCache(dim, heads, sum(-(-n // page) for n in lengths) + 2, page)
    for N, F in ((cache.k_N, cache.k_F), (cache.v_N, cache.v_F)):
        N.fill_(float("nan"))                                           # of what no sequence has
        F.fill_(77)
    tables, table, length_t = deal(cache, lengths, 301)
    for b, n in enumerate(lengths):
        if n == 0:
            continue
        j = np.arange(n)
        at = torch.from_numpy(np.asarray(tables[b])[j // page].astype(np.int64)).cuda()
        place = torch.from_numpy(j % page).cuda()
        for head in range(heads):
            low, F = code.lines(case, head, b)
            low = torch.from_numpy(low).cuda()
            cache.k_F[at, head, place] = 0
            cache.k_F[at, head, place, 0] = torch.where(low, -127, 0).to(torch.int8)
            cache.k_N[at, head, place] = torch.where(low, 100.0, 1.0)
            cache.v_F[at, head, place] = torch.from_numpy(F).cuda()
            cache.v_N[at, head, place] = 1.0
        for hole in holes:
            if hole < len(tables[b]):
                table[b, hole] = -1 - hole if hole % 2 else cache.n_pages + hole
    q = torch.full((sum(new), heads * groups, dim), code.query(dim), device="cuda", dtype=torch.float16)
    return cache, table, length_t, q


@pytest.mark.parametrize("longest", [0, 64, 500])
@pytest.mark.parametrize("name", sorted(code.CASES))
def test_each_position_once(name, longest):
    case = code.CASES[name]
    dim, heads, groups, page, lengths, new, causal, window, holes = case
    cache, table, length_t, q = coded(case)
    H = torch.from_numpy(matrix("dct", dim)).cuda()
    for most in sorted({1, max(new)}):
        lse = torch.full(q.shape[:2], 7.0, device="cuda")
        out = cache.attend(q, table, length_t, starts=starts_of(new), max_new=most, max_length=longest, causal=causal, window=window, scale=1.0,
                           lse=lse)
        got, got_lse = (out.double() @ H).cpu().numpy(), lse.double().cpu().numpy()
        first = 0
        for b, count in enumerate(new):
            for g in range(heads * groups):
                want, want_lse = code.expected(case, g // groups, b)
                error = np.linalg.norm(got[first:first + count, g] - want, axis=-1)
                empty = np.isneginf(want_lse)
                assert (error <= code.tolerance(want)).all(), (name, b, g, most, (error / code.tolerance(want)).max())
                assert (got[first:first + count, g][empty] == 0).all()
                mine, off = got_lse[first:first + count, g], want_lse.copy()
                assert np.isneginf(mine[empty]).all()
                off[empty] = 0
                assert (np.abs(mine - off) <= code.lse_tolerance(off))[~empty].all(), (name, b, g, most)
            first += count


# Single tokens whose query heads to a head of the cache are more than half a tile of 128: they take the kernel for many rows, without starts.
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("groups", [65, 128, 129, 300])
@pytest.mark.parametrize("lengths", [[200], [40, 0, 333], [2000, 5]])
def test_many_query_heads_to_a_head_of_the_cache(dim, groups, lengths):
    cache = filled(PagedCache(dim, 1, sum(-(-n // 32) for n in lengths) + 1, 32), 311, spread=False)
    tables, table, length_t = deal(cache, lengths, 312)
    g = torch.Generator(device="cuda").manual_seed(313)
    q = torch.randn(len(lengths), groups, dim, generator=g, device="cuda").to(torch.float16)
    for window in (0, 50):
        lse, again = torch.full(q.shape[:2], 7.0, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
        out = cache.attend(q, table, length_t, window=window, lse=lse)
        check_attend(cache, q, out, lse, tables, lengths, [1] * len(lengths), window=window)
        with_starts = cache.attend(q, table, length_t, starts=starts_of([1] * len(lengths)), max_new=1, window=window, lse=again)
        check_attend(cache, q, with_starts, again, tables, lengths, [1] * len(lengths), window=window)


# and the same in two heads of the cache whose results tell positions apart
@pytest.mark.parametrize("dim, groups, lengths", [(64, 65, [900]), (128, 129, [1500, 64, 1]), (256, 300, [700, 65])])
def test_many_query_heads_see_each_position_once(dim, groups, lengths):
    case = (dim, 2, groups, 32, lengths, [1] * len(lengths), True, 0, ())
    cache, table, length_t, q = coded(case)
    H = torch.from_numpy(matrix("dct", dim)).cuda()
    for longest in (0, 64):
        lse = torch.empty(q.shape[:2], device="cuda")
        got = (cache.attend(q, table, length_t, max_length=longest, scale=1.0, lse=lse).double() @ H).cpu().numpy()
        for b in range(len(lengths)):
            for head in range(2):
                want, want_lse = code.expected(case, head, b)
                rows = slice(head * groups, (head + 1) * groups)
                assert (np.linalg.norm(got[b, rows] - want, axis=-1) <= code.tolerance(want)).all()
                assert (np.abs(lse[b, rows].double().cpu().numpy() - want_lse) <= code.lse_tolerance(want_lse)).all()
