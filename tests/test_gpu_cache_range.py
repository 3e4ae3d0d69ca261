"""Attention over the paged cache where lines differ widely in size: every finite line, seen or not, leaves the rows what the definition says.

Tolerances are those of test_gpu_cache.py's check of a row, in which the weights' rounding is relative to what the row itself sees: sum_j p_j |v_j|.
Multiplying all N by a power of two is exact, and so is taking it off the results again.
"""
import math

import pytest
import torch

from paper_2406_11209_amd.cache import PagedCache
from test_gpu_cache import FLOATS, check_attend, deal, filled, starts_of

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

# dim, heads, groups, page, work, length, new tokens, max_length: rows by the few and by the many, one and several splits of the positions
SHAPES = [
    (128, 2, 4, 64, "f32", 200, 1, 0),              # 4 rows
    (128, 1, 1, 16, "bf16", 1500, 1, 0),
    (32, 1, 4, 16, "f32", 300, 9, 0),               # two tiles of rows
    (64, 1, 3, 32, "f32", 130, 20, 0),
    (32, 2, 4, 16, "bf16", 200, 100, 0),            # every wave with rows of its own
    (128, 1, 4, 64, "f32", 400, 100, 0),
    (128, 1, 2, 16, "f32", 257, 257, 64),           # positions not split
    (64, 2, 2, 16, "bf16", 3000, 120, 0),
    (256, 1, 4, 32, "f32", 90, 40, 0),
    (256, 1, 2, 32, "f32", 700, 3, 0),
]


def made(shape, seed, array):
    dim, heads, groups, page, work, length, new, longest = shape
    cache = filled(PagedCache(dim, heads, -(-length // page) + 1, page, work), seed, spread=False)
    tables, table, lengths = deal(cache, [length], seed + 1)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    q = torch.randn(new, heads * groups, dim, generator=g, device="cuda").to(FLOATS[array])
    return cache, tables, table, lengths, q


@pytest.mark.parametrize("array", ["bf16", "f16"])
@pytest.mark.parametrize("power", [12, 16, 24, 33, 60, 118])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_large_lines_that_a_row_does_not_see(shape, power, array):
    """A value 2^power times the others': later than a row, before its window, or further than its sequence reaches."""
    dim, heads, groups, page, work, length, new, longest = shape
    cache, tables, table, lengths, q = made(shape, 101, array)
    options = dict(starts=starts_of([new]), max_new=new, max_length=longest)

    def grown(position):
        cache.v_N[tables[0][position // page], :, position % page] *= 2.0 ** power

    def shrunk(position):
        cache.v_N[tables[0][position // page], :, position % page] *= 2.0 ** -power

    if new > 1:                                                          # seen by the last rows only
        own = new - max(1, new // 3)
        at = length - new + own
        grown(at)
        out = cache.attend(q, table, lengths, **options)
        check_attend(cache, q[:own], out[:own], None, tables, [at], [own])
        shrunk(at)
    window = max(3, min(length - new, 100))                             # seen by no row, or by the first ones
    at = length - new - window
    if at >= 0:
        grown(at)
        out = cache.attend(q, table, lengths, window=window, **options)
        check_attend(cache, q, out, None, tables, [length], [new], window=window)
        shrunk(at)
    if new > 2:
        at = length - new - window + 1 + new // 2                        # the first half of the rows sees it
        if 0 <= at < length - new:
            grown(at)
            out = cache.attend(q, table, lengths, window=window, **options)
            last = slice(new - (new - new // 2 - 1), new)
            check_attend(cache, q[last], out[last], None, tables, [length], [last.stop - last.start], window=window)
            shrunk(at)
    if length % page:                                                    # behind the end, in the last page
        grown(length)
        out = cache.attend(q, table, lengths, **options)
        check_attend(cache, q, out, None, tables, [length], [new])


@pytest.mark.parametrize("array", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_large_lines_of_vanishing_weight(shape, array):
    """A value 2^40 times the others' that every row sees, its key's score 2^-100 or less of the others' weights; and a value of zeros whose score is far
    ahead, beside which the others are all that counts."""
    dim, heads, groups, page, work, length, new, longest = shape
    for far, v_power in ((-120.0, 2.0 ** 40), (30.0, 0.0)):
        cache, tables, table, lengths, q = made(shape, 111, array)
        q[..., :] = 1 / math.sqrt(dim)                                   # coefficient 0 is 1 under the DCT, the others 0
        cache.k_F.fill_(0)
        cache.k_F[..., 0] = 127
        cache.k_N.fill_(1.0)
        for position in (0, (length - new) // 2):
            at = (tables[0][position // page], slice(None), position % page)
            cache.k_F[at + (0,)] = 127 if far > 0 else -127
            cache.k_N[at] = abs(far)
            cache.v_N[at] *= v_power
        if far > 0:
            cache.v_N.copy_(cache.v_N.double() * 2.0 ** 40)                 # so that their sum is not a small number
        out = cache.attend(q, table, lengths, starts=starts_of([new]), max_new=new, max_length=longest, scale=1.0)
        own = slice(1 if length == new else 0, new)                     # (a prompt's first row sees nothing else)
        check_attend(cache, q[own], out[own], None, tables, [length], [own.stop - own.start], scale=1.0)


@pytest.mark.parametrize("power", [-90, -50, 30, 100, 121])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_values_of_any_size(shape, power):
    """All values 2^power times as large: the results are, too."""
    dim, heads, groups, page, work, length, new, longest = shape
    cache, tables, table, lengths, q = made(shape, 121, "bf16")
    plain = cache.v_N.clone()
    cache.v_N.copy_(plain.double() * 2.0 ** power)
    out = cache.attend(q, table, lengths, starts=starts_of([new]), max_new=new, max_length=longest)
    cache.v_N.copy_(plain)
    check_attend(cache, q, out.double() * 2.0 ** -power, None, tables, [length], [new])


@pytest.mark.parametrize("power", [-90, 60, 95])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_keys_of_any_size(shape, power):
    """Keys 2^power times as large and queries as much smaller: the same scores; and a scale of 0, by which all weights are alike."""
    dim, heads, groups, page, work, length, new, longest = shape
    cache, tables, table, lengths, q = made(shape, 131, "bf16")
    plain = cache.k_N.clone()
    cache.k_N.copy_(plain.double() * 2.0 ** power)
    small = (q.double() * 2.0 ** -power).to(q.dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    options = dict(starts=starts_of([new]), max_new=new, max_length=longest)
    out = cache.attend(small, table, lengths, lse=lse, **options)
    none = cache.attend(q, table, lengths, scale=0.0, **options)
    cache.k_N.copy_(plain)
    check_attend(cache, q, out, lse, tables, [length], [new])
    check_attend(cache, q, none, None, tables, [length], [new], scale=0.0)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 9, 2 ** 30])
@pytest.mark.parametrize("dim, heads, groups", [(128, 2, 2), (32, 1, 4), (64, 1, 40), (256, 1, 3), (128, 1, 16)])
def test_windows_as_wide_as_they_come(dim, heads, groups, window):
    """More new tokens than positions put rows before position 0; a window that reaches past everything hides nothing."""
    for causal in (True, False):
        lengths_, counts = [5, 0, 40, 20], [9, 3, 40, 60]
        cache = filled(PagedCache(dim, heads, 8, 16), 141)
        tables, table, lengths = deal(cache, lengths_, 142)
        q = torch.randn(sum(counts), heads * groups, dim, device="cuda").to(torch.bfloat16)
        lse = torch.empty(q.shape[:2], device="cuda")
        out = cache.attend(q, table, lengths, starts=starts_of(counts), max_new=max(counts), causal=causal, window=window, lse=lse)
        check_attend(cache, q, out, lse, tables, lengths_, counts, causal)
        few = cache.attend(q[:12], table[:2], lengths[:2], starts=starts_of(counts[:2]), max_new=1, causal=causal, window=window)
        check_attend(cache, q[:12], few, None, tables[:2], lengths_[:2], counts[:2], causal)


@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_sums_of_values_near_the_end_of_the_range(shape):
    """Values whose mean FP32 holds, and whose sum it does not."""
    dim, heads, groups, page, work, length, new, longest = shape
    cache, tables, table, lengths, q = made(shape, 151, "bf16")
    cache.v_F.fill_(0)
    cache.v_F[..., 1] = torch.randint(90, 127, cache.v_F.shape[:-1], device="cuda").to(torch.int8)
    cache.v_N.fill_(2.0 ** 125)
    out = cache.attend(q * 0.1, table, lengths, starts=starts_of([new]), max_new=new, max_length=longest)
    cache.v_N.fill_(1.0)
    check_attend(cache, q * 0.1, out.double() * 2.0 ** -125, None, tables, [length], [new])


@pytest.mark.parametrize("low, high, share", [(-70, 100, 1.0), (-70, 100, 0.03), (-30, 60, 0.3), (10, 40, 0.1)])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{i}" for i in range(len(SHAPES))])
def test_lines_of_every_size(shape, low, high, share):
    """Values of any size between 2^low and 2^high among others of one, and some of zero, in any order, all of them seen."""
    dim, heads, groups, page, work, length, new, longest = shape
    cache, tables, table, lengths, q = made(shape, 161, "bf16")
    g = torch.Generator(device="cuda").manual_seed(162)
    powers = torch.randint(low, high + 1, cache.v_N.shape, generator=g, device="cuda").double()
    drawn = torch.rand(powers.shape, generator=g, device="cuda") < share
    lse = torch.empty(q.shape[:2], device="cuda")
    plain = cache.v_N.clone()
    for others in (low, high):
        cache.v_N.copy_(plain.double() * torch.exp2(torch.where(drawn, powers, float(others))))
        cache.v_N[torch.rand(powers.shape, generator=g, device="cuda") < 0.1] = 0
        out = cache.attend(q, table, lengths, starts=starts_of([new]), max_new=new, max_length=longest, lse=lse)
        check_attend(cache, q, out, lse, tables, [length], [new])
