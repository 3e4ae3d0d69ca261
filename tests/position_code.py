"""Caches in which every position that a row sees, or must not see, can be told from its result.

Keys are zero, or (a third of the positions, drawn at random) have a score of -100: what sees one of the former weighs them alike and the latter not
at all, exactly.  A value has 63 at two coefficients that say which position it is of, so that a result is a count of positions by two
digits of base D, over how many there are, and lse the logarithm of that.  Weights, products and sums are then exact; what is off is the transform back (2^-17
of the norm), FP16's rounding of the result (2^-11 of it, and 2^-25 an element below its normal numbers), and lse by FP32's logarithm.
"""
import math

import numpy as np

# dim, heads, groups, page, lengths, new tokens, causal, window, table columns that are holes
CASES = {
    "token-records": (128, 2, 4, 64, [3000], [1], True, 0, ()),
    "tokens-records": (128, 1, 2, 16, [2500, 1, 70], [1, 1, 1], True, 0, ()),
    "token-holes": (64, 1, 4, 16, [2000], [1], True, 0, (0, 4, 7, 63, 64)),
    "token-window": (64, 1, 5, 16, [2000, 60], [1, 1], True, 700, ()),
    "token-window-of-one": (128, 1, 5, 16, [200, 64], [1, 1], True, 1, ()),
    "two-row-waves-256": (256, 1, 8, 32, [2000, 70], [1, 3], True, 0, ()),
    "two-row-waves-128": (128, 1, 4, 32, [1000, 17], [12, 11], True, 0, (3,)),
    "few-rows-64": (64, 3, 1, 32, [1500, 129], [20, 17], True, 0, ()),
    "four-row-waves-32": (32, 2, 8, 16, [1000, 40], [60, 40], True, 0, (2, 40)),
    "four-row-waves-32-window": (32, 1, 8, 16, [700], [50], True, 65, ()),
    "many-rows-prompt": (128, 2, 4, 64, [513], [513], True, 0, ()),
    "many-rows-records": (128, 2, 4, 64, [3000], [64], True, 0, ()),
    "many-rows-few-heads": (128, 1, 8, 16, [2500, 0, 70, 31], [40, 5, 70, 40], True, 0, (1, 8, 77)),
    "many-rows-window": (64, 3, 2, 32, [2100, 200], [77, 130], True, 300, ()),
    "many-rows-window-of-one": (128, 1, 5, 128, [300], [300], True, 1, ()),
    "many-rows-all": (64, 1, 16, 16, [3000], [9], False, 0, ()),
    "many-rows-all-window": (64, 1, 8, 32, [100, 260], [100, 33], False, 20, ()),
    "many-rows-256": (256, 1, 4, 64, [2000, 129], [33, 129], True, 0, (16,)),
    "many-rows-256-window": (256, 2, 2, 1024, [900], [200], True, 64, ()),
}


def query(dim):
    """Elements of a query whose coefficients are 1 (but for FP16's rounding) and zeros, under the DCT."""
    return float(np.float16(dim ** -0.5))


def lines(case, head, b):
    """(which positions have a score of -100, F of values [length, D]) of a head of the cache and a sequence."""
    dim, length = case[0], case[4][b]
    rng = np.random.default_rng(1000 * head + b)
    low = rng.random(length) < 1 / 3
    F = np.zeros((length, dim), dtype=np.int8)
    j = np.arange(length)
    np.add.at(F, (j, (j + 5 * head) % dim), 63)
    np.add.at(F, (j, (j // dim * 37 + 11) % dim), 63)
    return low, F


def visible(case, b):
    """[new, length] of what the tokens of sequence b see."""
    page, length, new, causal, window, holes = case[3], case[4][b], case[5][b], *case[6:]
    at, j = np.arange(length - new, length)[:, None], np.arange(length)[None, :]
    seen = (j <= at) if causal else np.ones((new, length), dtype=bool)
    if window:
        seen = seen & (j > at - window)
    return seen & ~np.isin(j // page, holes)


def weighed(seen, low):
    """The positions that have all the weight, for every row."""
    high = seen & ~low
    return np.where(high.any(1, keepdims=True), high, seen)


def expected(case, head, b):
    """Coefficients of the results [new, D], and lse."""
    low, F = lines(case, head, b)
    w = weighed(visible(case, b), low)
    n = w.sum(1)
    sums = w.astype(np.float64) @ (F.astype(np.float64) / 127.0)
    with np.errstate(divide="ignore"):
        lse = np.log(n) - 100.0 * query(case[0]) * math.sqrt(case[0]) * (low[None, :] & w).any(1)
    return sums / np.maximum(n, 1)[:, None], lse


def tolerance(coefficients):
    """Of a result, in the norm."""
    dim = coefficients.shape[-1]
    return (2.0 ** -11 + 2.0 ** -17) * np.linalg.norm(coefficients, axis=-1) + 2.0 ** -25 * math.sqrt(dim)


def lse_tolerance(lse):
    return 2.0 ** -20 * (1 + np.abs(lse)) + (np.abs(lse) > 50) * 100 * 2.0 ** -16     # (a score of -100: the query's transform and fixed point)
