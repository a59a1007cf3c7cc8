"""Buckets.logarithmic: the interval and table row of every relative position, against the definition distance by distance."""
import math

import pytest

from paper_2308_09187_amd import qgx


def row_of(b, delta):
    n = b._c.n
    for i in range(n):
        if b._bounds[i] <= delta < b._bounds[i + 1]:
            return b._rows[i]
    return None


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("rows,far", [(32, 128), (8, 64), (16, 100), (64, 250), (4, 3), (128, 1000)])
def test_rows_follow_the_logarithm(rows, far, both):
    m = rows // 2 if both else rows
    exact = m // 2
    b = qgx.Buckets.logarithmic(rows, far, both)
    for n in range(0, 3 * far):
        if n < exact:
            want = {n}
        else:
            x = exact + (m - exact) * math.log(n / exact) / math.log(far / exact)
            # at a start the logarithm may fall on either side; several starts below one whole number leave rows without a distance
            want = {min(m - 1, math.floor(x + e)) for e in (-1e-9, 1e-9)}
        got = row_of(b, -n)
        if far > 4 * m:                                  # starts are further apart than one
            assert got in want, n
        assert got is not None and (n == 0 or got >= row_of(b, -(n - 1)))
        if both and n:
            assert row_of(b, n) == m + got
        if not both and n:
            assert row_of(b, n) is None
    assert row_of(b, -(1 << 29)) == m - 1


@pytest.mark.parametrize("both", [False, True])
def test_window(both):
    b = qgx.Buckets.logarithmic(16, 100, both, window=40)
    whole = qgx.Buckets.logarithmic(16, 100, both)
    for delta in range(-100, 101):
        assert row_of(b, delta) == (row_of(whole, delta) if abs(delta) < 40 else None)


def test_refusals():
    for args in ((1, 100), (2, 1), (32, 16)):
        with pytest.raises(qgx.QgxError):
            qgx.Buckets.logarithmic(*args)
    with pytest.raises(qgx.QgxError):
        qgx.Buckets.logarithmic(16, 100, window=0)
    with pytest.raises(qgx.QgxError):
        qgx.Buckets([0, 1], [0, 1])
