"""The cases that tell positions apart (position_code.py) do: a mistake planted in the expected result, at any one position of any row, is more than
the tolerance allows.  No GPU."""
import numpy as np
import pytest

import position_code as code


@pytest.mark.parametrize("name", sorted(code.CASES))
def test_every_position_counts(name):
    case = code.CASES[name]
    rng = np.random.default_rng(0)
    for b, (length, new) in enumerate(zip(case[4], case[5])):
        low, F = code.lines(case, 0, b)
        seen = code.visible(case, b)
        w = code.weighed(seen, low)
        want, _ = code.expected(case, 0, b)
        A = F.astype(np.float64) / 127.0
        rows = range(new) if new <= 12 else sorted({0, 1, new // 2, new - 1} | set(rng.integers(0, new, 8).tolist()))
        for i in rows:
            n = int(w[i].sum())
            mine = np.flatnonzero(w[i])
            if n == 0:
                continue
            allowed = 2 * code.tolerance(want[i])
            # one lost, or counted twice: lse
            assert np.log((n + 1) / n) > 2 * code.lse_tolerance(np.log(n))
            # one taken for another, near it or a tile, a stage or a page away: the result
            for apart in (1, -1, 4, 8, 16, -16, 32, 64, -64, 128, case[3], -case[3]):
                other = mine + apart
                inside = (other >= 0) & (other < length)
                inside[inside] &= ~w[i][other[inside]]
                if inside.any():
                    moved = np.linalg.norm(A[other[inside]] - A[mine[inside]], axis=1) / n
                    assert moved.min() > allowed, (name, b, i, apart, moved.min() / allowed)
            # the result of as many positions as it should be, one lost and another counted twice
            if n > 1:
                twice = np.linalg.norm(A[mine[1:]] - A[mine[:-1]], axis=1) / n
                assert twice.min() > allowed, (name, b, i, twice.min() / allowed)
