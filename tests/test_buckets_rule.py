"""Buckets.logarithmic against its rule in whole numbers, distance by distance, tables whose rows lie less than one distance apart among them:
distance n >= e = m // 2 takes row e + t with the largest t < m - e for which (n / e)^(m - e) >= (far / e)^t."""
import bisect

import pytest

from paper_2308_09187_amd import qgx


def row_of(b, delta):
    bounds = list(b._bounds)
    i = bisect.bisect_right(bounds, delta) - 1
    return b._rows[i] if 0 <= i < b._c.n else None


def rule(n, m, far):
    e = m // 2
    if n < e:
        return n
    t = 0
    while t + 1 < m - e and n ** (m - e) >= e ** (m - e - t - 1) * far ** (t + 1):
        t += 1
    return e + t


@pytest.mark.parametrize("window", [None, 5, 40, 300])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("rows,far", [(4, 3), (4, 64), (8, 64), (8, 128), (16, 64), (32, 64), (32, 128), (32, 250), (64, 64), (64, 100), (64, 128), (64, 250), (100, 60),
                                      (128, 65), (128, 100), (128, 128), (128, 1000)])
def test_every_distance(rows, far, both, window):
    m = rows // 2 if both else rows
    b = qgx.Buckets.logarithmic(rows, far, both, window=window)
    bounds = list(b._bounds)
    assert all(x < y for x, y in zip(bounds, bounds[1:])) and b._c.n == len(bounds) - 1 <= qgx.MAX_INTERVALS
    for n in (*range(0, 1200), 1 << 29):
        want = rule(n, m, far) if window is None or n < window else None
        assert row_of(b, -n) == want
        if n:
            assert row_of(b, n) == (m + want if both and want is not None else None)
