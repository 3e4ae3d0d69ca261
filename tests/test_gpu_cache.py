"""The paged compressed cache on the GPU against plain computation in 64 bits, at the sizes and contents where it can go wrong.

Tolerances, from the roundings that the operators are documented to make:

  append   indices are those of the definition except where r C / N is within 1e-9 of a rounding border (64-bit transforms
           differ by some 1e-13); N within half a step of its type.
  attend   per row, in the 2-norm over its D values.  The query row: D elements of half a step of 1/32639 of the largest,
           and an FP32 transform (2^-17 of the norm): a score's error is at most the error's norm times the key's norm times
           the scale, and FP32 products and sums of scores add 2^-21 of it; call the largest over what the row sees e.
           Weights then are off by 2 e relatively (numerator and denominator), by 2^-20 for the exponential and the FP32
           sums, and by 2^-11 from their rounding to FP16 (2^-21 where kept in two parts); the sum of weighted values is off by that
           times sum_j p_j |v_j|; transforming back costs 2^-17 of the norm, rounding to the type eps / 2 of it.
"""
import math

import numpy as np
import pytest
import torch

from paper_2406_11209_amd import api
from paper_2406_11209_amd.api import Codec
from paper_2406_11209_amd.cache import PagedCache

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

FLOATS = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def matrix(transform, n):
    """H[m][q], columns the basis functions."""
    if transform == "dct":
        m, q = np.arange(n)[:, None], np.arange(n)[None, :]
        return np.where(q == 0, math.sqrt(1 / n), math.sqrt(2 / n) * np.cos(math.pi * (2 * m + 1) * q / (2 * n)))
    if n == 1:
        return np.ones((1, 1))
    half = matrix(transform, n // 2)
    low = np.kron(half, [[1.0], [1.0]]) / math.sqrt(2)
    high = np.kron(np.eye(n // 2), [[1.0], [-1.0]]) / math.sqrt(2)
    return np.concatenate([low, high], axis=1)


def filled(cache, seed, spread=True):
    """Random N and F in every pool, F over its whole range."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    for N, F in ((cache.k_N, cache.k_F), (cache.v_N, cache.v_F)):
        size = torch.rand(N.shape, generator=g, device="cuda") * 3 + 0.1
        if spread:
            size *= torch.exp2(torch.randint(-6, 5, N.shape, generator=g, device="cuda").float())
        N.copy_(size.to(N.dtype))
        rough = torch.randn(F.shape, generator=g, device="cuda") * 40
        F.copy_(rough.round().clamp(-128, 127).to(torch.int8))
    return cache


def lines_of(cache, N, F, pages, length):
    """[heads, length, D] float64 coefficients."""
    page = torch.as_tensor(np.asarray(pages, dtype=np.int64), device="cuda")
    C = N[page].double()[..., None] * F[page].double() / 127.0
    return C.transpose(0, 1).reshape(cache.heads, -1, cache.head_dim)[:, :length]


def check_attend(cache, q, out, lse, tables, lengths, counts, causal=True, window=0, scale=None, hidden_pages=()):
    """Every row of out and lse against the definition; tables: page numbers per sequence."""
    D, groups = cache.head_dim, q.shape[1] // cache.heads
    H = torch.from_numpy(matrix(cache.codec.transform, D)).cuda()
    scale = 1 / math.sqrt(D) if scale is None else scale
    half_step = torch.finfo(q.dtype).eps / 2
    weight_step = 2.0 ** -21 if q.dtype == torch.float16 else 2.0 ** -11
    first = 0
    for b, (pages, length, fresh) in enumerate(zip(tables, lengths, counts)):
        rows = q[first:first + fresh].double()
        got, got_lse = out[first:first + fresh].double(), None if lse is None else lse[first:first + fresh].double()
        first += fresh
        if fresh == 0:
            continue
        qh = rows @ H                                                     # [fresh, q_heads, D]
        q_error = math.sqrt(D) * qh.abs().amax(-1) * 0.5 / 32639 + 2.0 ** -17 * qh.norm(dim=-1)
        j = torch.arange(length, device="cuda")[None, :]
        at = torch.arange(length - fresh, length, device="cuda")[:, None]
        seen = (j <= at) if causal else (j >= 0).expand(fresh, length)
        if window:
            seen = seen & (j > at - window)
        hidden = torch.tensor([p in hidden_pages for p in pages], device="cuda")
        if length and hidden.any():
            seen = seen & ~hidden[(j // cache.page_size)]
        safe = [0 if p in hidden_pages else p for p in pages]
        k, v = lines_of(cache, cache.k_N, cache.k_F, safe, length), lines_of(cache, cache.v_N, cache.v_F, safe, length)
        for g in range(q.shape[1]):
            kh, vh = k[g // groups], v[g // groups]
            s = torch.where(seen, scale * (qh[:, g] @ kh.t()), -math.inf)
            top = s.amax(-1, keepdim=True) if length else torch.full((fresh, 1), -math.inf, device="cuda", dtype=torch.float64)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            e = torch.where(seen, torch.exp(s - top), torch.zeros_like(s))
            total = e.sum(-1, keepdim=True)
            empty = total[:, 0] == 0
            p = e / torch.where(total == 0, torch.ones_like(total), total)
            vv = torch.where(seen.any(0)[:, None], vh, torch.zeros_like(vh))
            exact = p @ vv @ H.t()
            score_error = abs(scale) * torch.where(seen, q_error[:, g, None] * kh.norm(dim=-1)[None, :], 0.0).amax(-1) \
                if length else torch.zeros(fresh, device="cuda", dtype=torch.float64)
            score_error = score_error + 2.0 ** -21 * torch.where(seen, s.abs(), 0.0).amax(-1) if length else score_error
            spread = p @ vv.norm(dim=-1)
            bound = (2 * score_error + 2.0 ** -20 + weight_step) * spread + 2.0 ** -17 * spread + half_step * exact.norm(dim=-1) + \
                2.0 ** -24 * math.sqrt(D)                                 # subnormal results of FP16
            error = (got[:, g] - exact).norm(dim=-1)
            assert bool((error <= bound).all()), (b, g, float((error / bound).max()))
            assert bool((got[:, g][empty] == 0).all())
            if got_lse is not None:
                want = torch.log(total[:, 0]) + top[:, 0]
                assert bool((got_lse[:, g][empty] == -math.inf).all())
                ok = (got_lse[:, g] - want).abs() <= score_error + 2.0 ** -20 * (1 + want.abs())
                assert bool((ok | empty).all()), (b, g, "lse")


def deal(cache, lengths, seed):
    """Pages for sequences of these lengths, in random order; (tables as lists, table tensor, lengths tensor)."""
    rng = np.random.default_rng(seed)
    order = rng.permutation(cache.n_pages).tolist()
    tables = []
    for n in lengths:
        need = -(-n // cache.page_size)
        tables.append(order[:need])
        order = order[need:]
    width = max(1, max(len(t) for t in tables))
    rows = [t + [-1] * (width - len(t)) for t in tables]
    return (tables, torch.tensor(rows, dtype=torch.int32, device="cuda"),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"))


def starts_of(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")


# ---- append ----------------------------------------------------------------------------------------------------------

def check_append(cache, x, N, F, slots, N_before, F_before):
    H = torch.from_numpy(matrix(cache.codec.transform, cache.head_dim)).cuda()
    n_slots = cache.n_pages * cache.page_size
    want_N, want_F, border = N_before.double().clone(), F_before.double().clone(), torch.zeros(F.shape, dtype=torch.bool, device="cuda")
    for t, slot in enumerate(slots):
        if not 0 <= slot < n_slots:
            continue
        C = x[t].double() @ H
        top = C.abs().amax(-1, keepdim=True)
        r = torch.where(top > 0, 127 * C / torch.where(top > 0, top, torch.ones_like(top)), torch.zeros_like(C))
        at = (slot // cache.page_size, slice(None), slot % cache.page_size)
        want_N[at], want_F[at] = top[:, 0], r.round()
        border[at] = ((r - r.floor()) - 0.5).abs() < 1e-9
    wrong = (F.double() - want_F).abs()
    assert bool((wrong[~border] == 0).all()), int((wrong[~border] != 0).sum())
    assert bool((wrong[border] <= 1).all())
    step = torch.finfo(N.dtype).eps / 2 + 1e-12
    assert bool(((N.double() - want_N).abs() <= step * want_N.abs() + torch.finfo(N.dtype).tiny).all())


@pytest.mark.parametrize("dim, heads, page, array, work, transform, tokens", [
    (128, 8, 64, "bf16", "f32", "dct", 37), (64, 5, 16, "f32", "f16", "dct", 333), (32, 1, 16, "f16", "bf16", "haar", 1),
    (256, 2, 32, "f64", "f32", "dct", 19), (256, 3, 128, "bf16", "bf16", "haar", 65), (128, 1, 16, "f16", "f16", "haar", 16),
    (32, 7, 1024, "f32", "f32", "dct", 100), (64, 2, 256, "f64", "f32", "haar", 50)])
def test_append(dim, heads, page, array, work, transform, tokens):
    n_pages = tokens // page + 3
    cache = filled(PagedCache(dim, heads, n_pages, page, work, transform), 1)
    before = [p.clone() for p in cache.pools]
    g = torch.Generator(device="cuda").manual_seed(2)
    kv = (torch.randn(tokens, 2, heads, dim, generator=g, device="cuda", dtype=torch.float64) * 3).to(FLOATS[array])
    if tokens > 3:
        kv[1, 0] = 0                                               # a line of zeros
        kv[2, 1, :, 1:] = 0                                        # a line with one value
    slots = np.random.default_rng(3).permutation(n_pages * page)[:tokens]
    if tokens > 10:
        slots[4], slots[7], slots[9] = -1, n_pages * page, -(1 << 62)
    cache.append(kv[:, 0], kv[:, 1], torch.from_numpy(slots).cuda())       # strided: keys and values side by side
    torch.cuda.synchronize()
    check_append(cache, kv[:, 0], cache.k_N, cache.k_F, slots.tolist(), before[0], before[1])
    check_append(cache, kv[:, 1], cache.v_N, cache.v_F, slots.tolist(), before[2], before[3])


@pytest.mark.parametrize("array", ["bf16", "f32"])
def test_append_takes_any_alignment_and_broadcast_heads(array):
    cache = filled(PagedCache(64, 3, 4, 16), 4)
    before = [p.clone() for p in cache.pools]
    flat = torch.randn(11 * 211 + 8, device="cuda").to(FLOATS[array])
    k = flat[1:].as_strided((11, 3, 64), (211, 67, 1))             # odd strides, odd address
    v = flat[3:].as_strided((11, 3, 64), (211, 0, 1))              # one head for all
    slots = torch.arange(20, 31, device="cuda")
    cache.append(k, v, slots)
    check_append(cache, k, cache.k_N, cache.k_F, slots.tolist(), before[0], before[1])
    check_append(cache, v, cache.v_N, cache.v_F, slots.tolist(), before[2], before[3])


def test_append_agrees_with_compress_and_decompress_reads_it():
    cache = PagedCache(128, 2, 2, 16)
    x = torch.randn(32, 2, 128, device="cuda")
    cache.append(x, -x, torch.arange(32, device="cuda"))
    codec = Codec((128,), "f32", "i8")
    N, F = codec.compress(x.reshape(-1))
    mine_N, mine_F = cache.k_N.transpose(1, 2).reshape(-1), cache.k_F.transpose(1, 2).reshape(-1, 128)
    assert float((mine_N - N).abs().max() / N.max()) < 1e-6
    assert int((mine_F.int() - F.int()).abs().max()) <= 1 and float((mine_F != F).float().mean()) < 1e-3
    y = codec.decompress(cache.v_N.reshape(-1), cache.v_F.reshape(-1, 128), (64 * 128,)).view(2, 2, 16, 128)
    back = y.transpose(1, 2).reshape(32, 2, 128)
    # binning: at most N / 254 a coefficient, so sqrt(D) of that in the norm
    assert bool(((back + x).norm(dim=-1) <= 1.001 * math.sqrt(128) * x.norm(dim=-1) / 254).all())


def test_append_marks_lines_that_are_not_finite():
    cache = filled(PagedCache(64, 2, 2, 16), 5)
    x = torch.randn(3, 2, 64, device="cuda", dtype=torch.float32)
    x[0, 1, 5], x[2, 0, 63] = math.nan, -math.inf
    cache.append(x, torch.ones_like(x), torch.tensor([3, 17, 20], device="cuda"))
    assert math.isnan(cache.k_N[0, 1, 3]) and math.isnan(cache.k_N[1, 0, 4])
    assert bool((cache.k_F[0, 1, 3] == 0).all()) and bool((cache.k_F[1, 0, 4] == 0).all())
    assert bool(torch.isfinite(cache.k_N[0, 0, 3])) and bool(torch.isfinite(cache.v_N).all())


@pytest.mark.parametrize("dim, transform", [(32, "dct"), (64, "haar"), (128, "dct"), (256, "dct")])
def test_append_of_quotients_on_the_borders(dim, transform):
    """127 C / N half-way between two indices, as near as FP64 comes: either of the two.  Next to that, by 2^-20 of a step, the nearer one."""
    H = torch.from_numpy(matrix(transform, dim)).cuda()
    k = torch.arange(dim, device="cuda", dtype=torch.float64) % 126
    for away in (0.0, 2.0 ** -20, -2.0 ** -20):
        C = (k + 0.5 + away) / 127.0
        C[0] = 1.0                                                      # N
        C = torch.stack([C, -C, 3.0 * C])[:, None]
        cache = PagedCache(dim, 1, 1, 16, transform=transform)
        cache.append(C @ H.t(), C @ H.t(), torch.arange(3, device="cuda"))
        for F in (cache.k_F, cache.v_F):
            r = 127.0 * C / C.abs().amax(-1, keepdim=True)
            off = (F[0, 0, :3, None].double() - r).abs()
            assert bool((off <= 0.5 + 1e-9).all()) and bool((F[0, 0, :3, 0].abs() == 127).all())


# ---- attend ----------------------------------------------------------------------------------------------------------

CASES = [
    # dim, heads, groups, page, array, work, transform, lengths, new tokens, causal, window
    (128, 2, 4, 64, "bf16", "f32", "dct", [1], [1], True, 0),
    (128, 2, 4, 16, "f16", "f16", "haar", [1, 15, 16, 17, 63, 64, 65], [1] * 7, True, 0),
    (64, 3, 1, 32, "bf16", "bf16", "dct", [127, 128, 129, 500], [1, 2, 16, 17], True, 0),
    (32, 1, 3, 16, "f16", "f32", "dct", [33, 48, 200], [33, 11, 0], True, 0),
    (32, 5, 16, 128, "bf16", "f32", "haar", [1000, 3], [1, 3], True, 0),
    (256, 1, 8, 32, "bf16", "f16", "dct", [700, 5, 64], [1, 5, 9], True, 0),
    (256, 2, 3, 16, "f16", "bf16", "haar", [130, 97], [70, 1], True, 0),
    (128, 1, 7, 64, "bf16", "f32", "dct", [3000], [1], True, 0),              # many splits
    (128, 1, 2, 16, "f16", "f32", "dct", [2500, 1], [1, 1], True, 0),
    (64, 2, 2, 64, "bf16", "f32", "dct", [300, 10], [300, 10], True, 0),      # whole prompts
    (128, 2, 4, 64, "bf16", "f32", "dct", [513], [513], True, 0),
    (128, 2, 4, 64, "f16", "f32", "haar", [400, 90], [100, 90], True, 37),    # windows
    (64, 1, 5, 16, "bf16", "f16", "dct", [2000, 60], [1, 33], True, 1),
    (64, 1, 5, 16, "f16", "f32", "dct", [2000, 2000], [1, 50], True, 700),
    (128, 2, 2, 32, "bf16", "f32", "dct", [100, 260], [100, 33], False, 0),   # every position seen
    (64, 1, 1, 32, "f16", "f32", "haar", [100, 260], [100, 33], False, 20),
    (64, 2, 2, 16, "bf16", "f32", "dct", [0, 5, 0, 20], [3, 9, 0, 20], True, 0),   # more new tokens than positions: empty rows
    (128, 1, 1, 16, "f16", "f32", "dct", [0], [2], False, 0),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{i}" for i in range(len(CASES))])
def test_attend(case):
    dim, heads, groups, page, array, work, transform, lengths, counts, causal, window = case
    n_pages = sum(-(-n // page) for n in lengths) + 2
    cache = filled(PagedCache(dim, heads, n_pages, page, work, transform), 7)
    tables, table, length_t = deal(cache, lengths, 8)
    # whatever no sequence owns, or lies past a sequence's end, is poison
    owned = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    for t, n in zip(tables, lengths):
        for i, p in enumerate(t):
            owned[p, :max(0, min(page, n - i * page))] = True
    for N in (cache.k_N, cache.v_N):
        N.masked_fill_(~owned[:, None, :], math.nan)
    g = torch.Generator(device="cuda").manual_seed(9)
    q = torch.randn(sum(counts), heads * groups, dim, generator=g, device="cuda")
    q = (q * torch.exp2(torch.randint(-3, 2, q.shape[:2], generator=g, device="cuda").float())[..., None]).to(FLOATS[array])
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = cache.attend(q, table, length_t, starts=starts_of(counts), max_new=max(counts), causal=causal, window=window, lse=lse)
    torch.cuda.synchronize()
    check_attend(cache, q, out, lse, tables, lengths, counts, causal, window)
    if all(c == 1 for c in counts):                  # the form without starts is the same call
        assert torch.equal(cache.attend(q, table, length_t, causal=causal, window=window), out)
    # bounds that are too low or too high only deal the work out otherwise
    for most, longest in ((1, 64), (5000, 0)):
        again = cache.attend(q, table, length_t, starts=starts_of(counts), max_new=most, max_length=longest, causal=causal,
                             window=window)
        check_attend(cache, q, again, None, tables, lengths, counts, causal, window)


# chunks of many rows, with and without splits of the positions: dim, heads, groups, page, array, work, transform, lengths, new, causal, window
TALL = [
    (128, 2, 4, 64, "bf16", "f32", "dct", [6000], [64], True, 0),
    (128, 1, 8, 16, "f16", "bf16", "haar", [2500, 0, 70, 31], [40, 5, 70, 40], True, 0),
    (64, 3, 2, 32, "bf16", "f16", "dct", [4100, 200], [77, 130], True, 300),
    (64, 1, 16, 16, "f16", "f32", "haar", [3000], [9], False, 0),
    (256, 1, 4, 64, "f16", "f16", "dct", [2000, 129], [33, 129], True, 0),
    (256, 2, 2, 1024, "bf16", "f32", "haar", [900], [200], True, 64),
    (32, 2, 8, 16, "bf16", "f32", "dct", [1500, 40], [60, 40], True, 0),
    (128, 1, 5, 128, "bf16", "bf16", "dct", [1300], [300], True, 1),
]


@pytest.mark.parametrize("case", TALL, ids=[f"{i}" for i in range(len(TALL))])
def test_attend_many_rows_with_holes(case):
    """Pages outside the pool among the sequences', poison in everything that no row may see."""
    dim, heads, groups, page, array, work, transform, lengths, counts, causal, window = case
    n_pages = sum(-(-n // page) for n in lengths) + 2
    cache = filled(PagedCache(dim, heads, n_pages, page, work, transform), 41)
    tables, table, length_t = deal(cache, lengths, 42)
    owned = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    hidden = (n_pages, -3)
    for b, (t, n) in enumerate(zip(tables, lengths)):
        for i in range(len(t)):
            if i % 5 == 2:
                t[i] = hidden[i % 2]
                table[b, i] = t[i]
            else:
                owned[t[i], :max(0, min(page, n - i * page))] = True
    for N in (cache.k_N, cache.v_N):
        N.masked_fill_(~owned[:, None, :], math.inf)
    g = torch.Generator(device="cuda").manual_seed(43)
    q = torch.randn(sum(counts), heads * groups, dim, generator=g, device="cuda").to(FLOATS[array])
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    for most, longest in ((max(counts), 0), (max(counts), 128), (1, 0)):
        out = cache.attend(q, table, length_t, starts=starts_of(counts), max_new=most, max_length=longest, causal=causal,
                           window=window, lse=lse)
        check_attend(cache, q, out, lse, tables, lengths, counts, causal, window, hidden_pages=hidden)


def test_rows_of_no_sequence_are_zero_beside_many_rows():
    cache = filled(PagedCache(128, 2, 12, 64), 44)
    tables, table, lengths = deal(cache, [200, 100], 45)
    q = torch.randn(200, 8, 128, device="cuda").to(torch.bfloat16)
    starts = torch.tensor([11, 111, 190], dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device="cuda")
    cache.attend(q, table, lengths, starts=starts, max_new=100, out=out, lse=lse)
    assert bool((out[:11] == 0).all()) and bool((out[190:] == 0).all())
    assert bool((lse[:11] == -math.inf).all()) and bool((lse[190:] == -math.inf).all())
    check_attend(cache, q[11:190], out[11:190], lse[11:190], tables, [200, 100], [100, 79])


# short enough for one workgroup to see every position of its rows, which then writes their results itself; row tiles to a workgroup 1, 2 and more
SHORT = [
    (32, 2, 4, 16, "f16", "f32", "haar", [100], [60], True, 0),
    (32, 4, 3, 32, "bf16", "bf16", "dct", [64, 9, 0], [40, 9, 2], True, 0),
    (64, 12, 2, 16, "bf16", "f32", "dct", [90, 250, 1], [20, 3, 1], True, 40),
    (64, 1, 64, 64, "f16", "f16", "dct", [100], [1], True, 0),
    (128, 16, 3, 16, "f16", "f32", "dct", [31, 200], [11, 13], False, 0),
    (128, 4, 4, 64, "bf16", "f16", "haar", [250, 100, 17], [1, 4, 8], True, 0),
    (256, 3, 8, 32, "bf16", "f32", "dct", [100, 40], [4, 1], True, 0),
    (256, 1, 12, 16, "f16", "bf16", "haar", [60, 120], [1, 4], True, 33),
]


@pytest.mark.parametrize("case", SHORT, ids=[f"{i}" for i in range(len(SHORT))])
def test_attend_short_sequences_of_few_rows(case):
    dim, heads, groups, page, array, work, transform, lengths, counts, causal, window = case
    cache = filled(PagedCache(dim, heads, sum(-(-n // page) for n in lengths) + 1, page, work, transform), 61)
    tables, table, length_t = deal(cache, lengths, 62)
    g = torch.Generator(device="cuda").manual_seed(63)
    before, behind = 2, 3                                                # rows of no sequence
    q = torch.randn(before + sum(counts) + behind, heads * groups, dim, generator=g, device="cuda").to(FLOATS[array])
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device="cuda")
    cache.attend(q, table, length_t, starts=starts_of(counts) + before, max_new=max(counts), causal=causal, window=window, out=out, lse=lse)
    own = slice(before, before + sum(counts))
    check_attend(cache, q[own], out[own], lse[own], tables, lengths, counts, causal, window)
    for rest in (slice(0, before), slice(before + sum(counts), None)):
        assert bool((out[rest] == 0).all()) and bool((lse[rest] == -math.inf).all())


def test_rows_of_no_sequence_are_zero_beside_split_positions():
    cache = filled(PagedCache(128, 3, 60, 64), 64)
    tables, table, lengths = deal(cache, [3000, 500], 65)
    q = torch.randn(12, 6, 128, device="cuda").to(torch.bfloat16)
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device="cuda")
    cache.attend(q, table, lengths, starts=torch.tensor([5, 6, 9], dtype=torch.int32, device="cuda"), max_new=3, out=out, lse=lse)
    for rest in (slice(0, 5), slice(9, None)):
        assert bool((out[rest] == 0).all()) and bool((lse[rest] == -math.inf).all())
    check_attend(cache, q[5:9], out[5:9], lse[5:9], tables, [3000, 500], [1, 3])


def test_queries_beyond_the_range_of_their_transform():
    """A row whose coefficients overflow FP32 is not finite; its neighbours are what they are without it."""
    cache = filled(PagedCache(128, 2, 4, 64), 66)
    tables, table, lengths = deal(cache, [100, 130], 67)
    q = torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16)
    q[0, 3] = 3e38
    out = cache.attend(q, table, lengths)
    assert not bool(torch.isfinite(out[0, 3].float()).any())
    q[0, 3] = 0
    assert torch.equal(cache.attend(q, table, lengths)[0, [0, 1, 2, 4, 5, 6, 7]], out[0, [0, 1, 2, 4, 5, 6, 7]])
    assert torch.equal(cache.attend(q, table, lengths)[1], out[1])


def test_values_that_widen_late():
    """The largest N of the values at the end of a long sequence, tiny ones before."""
    for dtype in (torch.bfloat16, torch.float16):
        cache = filled(PagedCache(128, 1, 20, 64), 46, spread=False)
        tables, table, lengths = deal(cache, [1200], 47)
        for i, p in enumerate(tables[0]):
            cache.v_N[p] *= 2.0 ** (i - 12)
        q = torch.randn(100, 2, 128, device="cuda").to(dtype)
        out = cache.attend(q, table, lengths, starts=starts_of([100]))
        check_attend(cache, q, out, None, tables, [1200], [100])
        one = cache.attend(q[-1:], table, lengths)
        check_attend(cache, q[-1:], one, None, tables, [1200], [1])


def test_attend_takes_any_alignment():
    cache = filled(PagedCache(64, 2, 12, 16), 11)
    tables, table, lengths = deal(cache, [40, 100], 12)
    flat = torch.randn(9 * 331 + 8, device="cuda").to(torch.bfloat16)
    q = flat[1:].as_strided((9, 4, 64), (331, 71, 1))
    room = torch.full((9 * 400 + 8,), 5.0, device="cuda", dtype=torch.bfloat16)
    out = room[3:].as_strided((9, 4, 64), (400, 77, 1))
    wide = torch.full((2, table.shape[1] + 3), 99, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    cache.attend(q, wide[:, :table.shape[1]], lengths, starts=starts_of([4, 5]), out=out)
    check_attend(cache, q, out, None, tables, [40, 100], [4, 5])
    rest = room.clone()
    rest[3:].as_strided((9, 4, 64), (400, 77, 1)).fill_(5.0)
    assert bool((rest == 5.0).all())                 # nothing else was written


def test_attend_hides_pages_outside_the_pool():
    cache = filled(PagedCache(128, 2, 12, 16), 13)
    tables, table, lengths = deal(cache, [75, 50], 14)
    table[0, 1], table[0, 4], table[1, 0] = 12, -7, 2 ** 31 - 1
    tables[0][1], tables[0][4], tables[1][0] = 12, -7, 2 ** 31 - 1
    q = torch.randn(8, 4, 128, device="cuda").to(torch.bfloat16)
    lse = torch.empty(8, 4, device="cuda")
    out = cache.attend(q, table, lengths, starts=starts_of([6, 2]), lse=lse)
    check_attend(cache, q, out, lse, tables, [75, 50], [6, 2], hidden_pages=(12, -7, 2 ** 31 - 1))
    gone = cache.attend(q, torch.full_like(table, -1), lengths, starts=starts_of([6, 2]), lse=lse)
    assert bool((gone == 0).all()) and bool((lse == -math.inf).all())


def test_attend_cuts_lengths_and_starts_to_what_there_is():
    cache = filled(PagedCache(64, 1, 4, 16), 15)
    tables, table, lengths = deal(cache, [32, 32], 16)
    q = torch.randn(6, 2, 64, device="cuda").to(torch.float16)
    want = cache.attend(q, table, lengths, starts=starts_of([3, 3]))
    far = torch.tensor([0, 3, 1000], dtype=torch.int32, device="cuda")
    assert torch.equal(cache.attend(q, table, lengths + 500, starts=far), want)
    none = cache.attend(q, table, lengths * 0 - 5, starts=starts_of([3, 3]))
    assert bool((none == 0).all())
    part = cache.attend(q, table, lengths, starts=torch.tensor([2, 3, 4], dtype=torch.int32, device="cuda"))
    assert bool((part[:2] == 0).all()) and bool((part[4:] == 0).all()) and bool((part[2:4] != 0).any())


def test_hidden_lines_that_are_not_finite_do_not_reach_the_result():
    for value in (math.nan, math.inf):
        cache = filled(PagedCache(128, 1, 8, 16), 17)
        tables, table, lengths = deal(cache, [80], 18)
        q = torch.randn(20, 4, 128, device="cuda").to(torch.bfloat16)          # positions 60 .. 79
        for N in (cache.k_N, cache.v_N):
            N[tables[0][4], 0, 70 - 64] = value                               # position 70: rows 10 .. 19 see it
        out = cache.attend(q, table, lengths, starts=starts_of([20]))
        assert bool(torch.isfinite(out[:10]).all())
        assert not bool(torch.isfinite(out[10:].float()).all(-1).any())
        clean = filled(PagedCache(128, 1, 8, 16), 17)
        check_attend(clean, q[:10], out[:10], None, tables, [70], [10])
        seen = cache.attend(q[10:11], table, torch.tensor([71], dtype=torch.int32, device="cuda"), window=1)    # nothing else in sight
        assert not bool(torch.isfinite(seen.float()).any())
    cache = filled(PagedCache(64, 1, 2, 16), 19)
    tables, table, lengths = deal(cache, [9], 20)
    q = torch.randn(2, 2, 64, device="cuda").to(torch.float16)
    q[1, 0, 3] = math.nan
    out = cache.attend(q, table, lengths, starts=starts_of([2]))
    assert bool(torch.isnan(out[1, 0]).all()) and bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(out[1, 1]).all())


def test_far_apart_scores_and_small_values_keep_their_weight():
    """One key far ahead of thousands whose values are far larger than its own: their sum is what counts."""
    cache = PagedCache(64, 1, 70, 64)
    n, D = 4096, 64
    cache.k_F.fill_(0)
    cache.v_F.fill_(0)
    cache.k_F[..., 0] = 127
    cache.k_N.fill_(1.0)
    cache.v_F[..., 1] = torch.randint(50, 127, cache.v_F.shape[:-1], device="cuda").to(torch.int8)
    cache.v_N.fill_(1.0)
    tables, table, lengths = deal(cache, [n], 21)
    cache.k_N[tables[0][0], 0, 0] = 12.0                  # e^11 ahead of each of the others
    cache.v_N[tables[0][0], 0, 0] = 1e-4
    for dtype in (torch.float16, torch.bfloat16):
        q = torch.full((1, 1, D), 1 / math.sqrt(D), device="cuda").to(dtype)    # coefficient 0 is 1 under the DCT
        out = cache.attend(q, table, lengths, scale=1.0)
        check_attend(cache, q, out, None, tables, [n], [1], scale=1.0)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attend_scales(scale):
    cache = filled(PagedCache(64, 1, 12, 16), 23, spread=False)
    tables, table, lengths = deal(cache, [150], 24)
    q = torch.randn(3, 2, 64, device="cuda").to(torch.float16) * 0.2
    out = cache.attend(q, table, lengths, starts=starts_of([3]), scale=scale)
    check_attend(cache, q, out, None, tables, [150], [3], scale=scale)


def test_attend_of_a_pool_past_32_bits():
    """Lines past 2^31 bytes of F: the last pages of a pool of 4.5 GiB."""
    page, heads, dim = 1024, 32, 128
    n_pages = (9 << 29) // (page * heads * dim) + 1
    k_F = torch.empty(n_pages, heads, page, dim, dtype=torch.int8, device="cuda")
    N = torch.full((n_pages, heads, page), 0.5, device="cuda")
    cache = PagedCache(dim, heads, n_pages, page, pools=(N, k_F, N.clone(), k_F))
    g = torch.Generator(device="cuda").manual_seed(25)
    last = n_pages - 1
    k_F[last] = torch.randint(-127, 128, k_F.shape[1:], generator=g, device="cuda").to(torch.int8)
    q = torch.randn(2, heads, dim, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.tensor([[last]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([700], dtype=torch.int32, device="cuda")
    out = cache.attend(q, table, lengths, starts=starts_of([2]))
    check_attend(cache, q, out, None, [[last]], [700], [2])
    x = torch.randn(1, heads, dim, generator=g, device="cuda")
    slot = torch.tensor([last * page + 900], device="cuda")
    cache.append(x, x, slot)
    H = torch.from_numpy(matrix("dct", dim)).cuda()
    C = x[0].double() @ H
    assert bool((k_F[last, :, 900].double() - 127 * C / C.abs().amax(-1, keepdim=True)).abs().max() <= 0.5 + 1e-6)


# ---- pages -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dim, heads, page, work, pairs", [(32, 1, 16, "f16", 1), (128, 8, 64, "f32", 5), (64, 3, 16, "bf16", 300),
                                                           (256, 2, 128, "f32", 31), (32, 1, 16, "f32", 257)])
def test_copy_pages(dim, heads, page, work, pairs):
    n_pages = 2 * pairs + 3
    cache = filled(PagedCache(dim, heads, n_pages, page, work), 27)
    picked = np.random.default_rng(28).permutation(n_pages)[:2 * pairs].reshape(pairs, 2)
    if pairs > 2:
        picked[1, 0] = picked[0, 0]                  # read twice
    want = [p.clone() for p in cache.pools]
    for w in want:
        w[picked[:, 1]] = w[picked[:, 0]]
    cache.copy_pages(picked)
    for got, w in zip(cache.pools, want):
        assert torch.equal(got, w)


@pytest.mark.parametrize("n_pages, n_pairs", [(65536, 897), (65537, 449), (65600, 3)])
def test_copy_pages_of_pools_of_many_pages(n_pages, n_pairs):
    """Pages' numbers of 16 bits and of more, in more pairs than a launch takes."""
    cache = filled(PagedCache(32, 1, n_pages, 16, "f16"), 71)
    order = np.random.default_rng(72).permutation(n_pages)[:2 * n_pairs].astype(np.int32)
    order[order == n_pages - 1] = order[0]
    order[0] = n_pages - 1
    pairs = order.reshape(-1, 2)
    want = [p.clone() for p in cache.pools]
    for pool in want:
        pool[torch.from_numpy(pairs[:, 1].copy()).cuda().long()] = pool[torch.from_numpy(pairs[:, 0].copy()).cuda().long()]
    cache.copy_pages(pairs)
    for pool, expected in zip(cache.pools, want):
        assert torch.equal(pool, expected)


def test_sequences_forked_written_and_compacted():
    """Sequences as a program uses them, against the lines kept aside in plain tensors."""
    cache = PagedCache(64, 2, 40, 16, "f32")
    g = torch.Generator(device="cuda").manual_seed(29)
    held = {}

    def write(seqs, counts):
        k, v = (torch.randn(sum(counts), 2, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        cache.extend_and_append(seqs, counts, k, v)
        first = 0
        for s, n in zip(seqs, counts):
            held[s] = tuple(torch.cat([held[s][i], x[first:first + n]]) for i, x in enumerate((k, v)))
            first += n

    def check(seqs, counts):
        q = torch.randn(sum(counts), 4, 64, generator=g, device="cuda").to(torch.bfloat16)
        out = cache.attend_sequences(seqs, counts, q)
        check_attend(cache, q, out, None, [cache.pages.table(s).tolist() for s in seqs], [cache.length(s) for s in seqs], counts)
        for s in seqs:                               # what the pages hold is what was written
            k = lines_of(cache, cache.k_N, cache.k_F, cache.pages.table(s).tolist(), cache.length(s)) @ \
                torch.from_numpy(matrix("dct", 64)).cuda().t()
            x = held[s][0].double().transpose(0, 1)
            assert bool(((k - x).norm(dim=-1) <= 1.001 * 8 * x.norm(dim=-1) / 254).all())

    nothing = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    a, b = cache.open(), cache.open()
    held[a] = held[b] = (nothing, nothing)
    write([a, b], [37, 20])
    check([a, b], [37, 5])
    c = cache.fork(a)
    held[c] = held[a]
    write([a, c], [3, 9])                            # both write into the page they share
    check([a, b, c], [1, 1, 9])
    cache.close(b)
    del held[b]
    assert cache.compact() > 0
    check([c, a], [2, 3])
    cache.truncate(c, 30)
    held[c] = tuple(x[:30] for x in held[c])
    write([c], [25])
    check([a, c], [4, 25])
    free = cache.pages.free_count
    with pytest.raises(api.PbzError):                # too long for the pool: nobody is any longer than before
        cache.extend_and_append([a, c], [1, 700], torch.zeros(701, 2, 64, device="cuda"), torch.zeros(701, 2, 64, device="cuda"))
    assert cache.pages.free_count >= free - 1
    check([a, c], [4, 25])


def test_refusals_of_the_binding():
    cache = PagedCache(64, 2, 4, 16)
    x = torch.zeros(3, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.arange(3, device="cuda")
    bad = [lambda: cache.append(x, x, slots.int()), lambda: cache.append(x, x[:2], slots), lambda: cache.append(x, x.float(), slots),
           lambda: cache.append(x.cpu(), x, slots), lambda: cache.append(x[:, :1], x, slots), lambda: cache.append(x, x, slots.cpu()),
           lambda: cache.append(x.transpose(1, 2).contiguous().transpose(1, 2), x, slots), lambda: cache.append(x.int(), x.int(), slots)]
    table, lengths = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    bad += [lambda: cache.attend(x, table.long(), lengths), lambda: cache.attend(x, table[:2], lengths),
            lambda: cache.attend(x, table, lengths.long()), lambda: cache.attend(x[0], table, lengths),
            lambda: cache.attend(x, table, lengths, out=x.float()), lambda: cache.attend(x, table, lengths, out=x[:2]),
            lambda: cache.attend(x, table, lengths, starts=torch.zeros(3, dtype=torch.int32, device="cuda")),
            lambda: cache.attend(x, table, lengths, lse=torch.zeros(3, 2, device="cuda", dtype=torch.float64)),
            lambda: PagedCache(64, 2, 4, 16, pools=[p[:3] for p in cache.pools])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    for call, status in ((lambda: cache.attend(x.float(), table, lengths), -4), (lambda: cache.attend(x, table, lengths, window=-1), -7),
                         (lambda: cache.attend(x[:, :1], table, lengths), -7), (lambda: cache.attend(x[:2], table, lengths), -7),
                         (lambda: cache.attend(x, table, lengths, scale=math.nan), -9), (lambda: cache.copy_pages([(0, 4)]), -15),
                         (lambda: cache.attend(x, table, lengths, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), -8)):
        with pytest.raises(api.PbzError) as e:
            call()
        assert e.value.status == status
    empty = x[:0]
    cache.append(empty, empty, slots[:0])
    assert cache.attend(empty, table, lengths, starts=torch.zeros(4, dtype=torch.int32, device="cuda")).shape == (0, 2, 64)


# ---- streams and graphs ----------------------------------------------------------------------------------------------

def test_on_a_stream_of_its_own():
    cache = filled(PagedCache(128, 2, 40, 16), 31)
    tables, table, lengths = deal(cache, [300, 200], 32)
    q = torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16)
    want = cache.attend(q, table, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cache.attend(q, table, lengths)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_captured_step():
    """One decoding step, append and attend, as a graph that is replayed with other contents."""
    cache = filled(PagedCache(128, 2, 40, 16), 33)
    tables, table, lengths = deal(cache, [300, 200], 34)
    k, v, q = (torch.zeros(2, h, 128, device="cuda", dtype=torch.bfloat16) for h in (2, 2, 8))
    slots = torch.tensor([t[(n - 1) // 16] * 16 + (n - 1) % 16 for t, n in zip(tables, [300, 200])], device="cuda")
    out, space = torch.empty_like(q), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def step():
        cache.append(k, v, slots)
        cache.attend(q, table, lengths, out=out, workspace=space)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, device="cuda"))
        if i == 2:
            lengths.sub_(40)                          # shorter sequences, tokens to other slots
            slots.copy_(torch.tensor([t[(n - 1) // 16] * 16 + (n - 1) % 16 for t, n in zip(tables, [260, 160])], device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        replayed, pools = out.clone(), [p.clone() for p in cache.pools]
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed)
        for p, r in zip(cache.pools, pools):
            assert torch.equal(p, r)
        n = lengths.tolist()
        check_attend(cache, q, out, None, [t[:-(-m // 16)] for t, m in zip(tables, n)], n, [1, 1])


def test_the_example_layer():
    """The example's layer on a compressed cache against the same one uncompressed.  Binning moves a coefficient by up to N / 254, a key or value
    by up to sqrt(D) N / 254, which for the example's normal lines (N about 3 of a norm of sqrt(D)) is 3 sqrt(128) / 254 = 0.13 of its norm at most and
    a third of that (uniform) on the whole: 0.05 for values and, through scores of that much, less for weights."""
    from paper_2406_11209_amd.examples import paged_cache
    assert paged_cache.main(tokens=300, steps=3) < 0.13
