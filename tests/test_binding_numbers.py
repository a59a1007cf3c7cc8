"""Numbers that the C side's fields do not hold are refused by the binding (ctypes itself would take them modulo 2^32 or 2^64)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2308_09187_amd import qgx  # noqa: E402

LOW, HIGH = -(1 << 31), (1 << 31) - 1


def refused(f):
    with pytest.raises(qgx.QgxError) as e:
        f()
    assert e.value.status == qgx.ERR_ARG and str(e.value)


def test_bounds_and_rows_of_buckets():
    for bounds, rows in (([LOW - 1, 0], [0]), ([0, HIGH + 1], [0]), ([-(1 << 32), 1], [0]), ([0, (1 << 32) + 1], [0]), ([0, 1], [1 << 32]), ([0, 1], [-1])):
        refused(lambda: qgx.Buckets(bounds, rows))
    b = qgx.Buckets([LOW, 0, HIGH], [(1 << 32) - 1, 0])
    assert list(b._bounds) == [LOW, 0, HIGH] and list(b._rows) == [(1 << 32) - 1, 0]


@pytest.mark.parametrize("both", [False, True])
def test_a_window_wider_than_any_distance(both):
    for window in (HIGH, 1 << 31, 1 << 32, (1 << 40) + 7):
        b = qgx.Buckets.logarithmic(16, 100, both, window=window)
        assert list(b._bounds) == sorted(set(b._bounds)) and b._bounds[0] < -3 << 29
        assert b._bounds[b._c.n] == 1 if not both else b._bounds[b._c.n] > 3 << 29


@pytest.mark.gpu
def test_offsets():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = qgx.Context(64, 2, 256)
    x = torch.zeros(2, 10, device="cuda")
    for off in (65, 1 << 32, 1 << 64, (1 << 64) + 4, -1, -(1 << 64)):
        refused(lambda: c.tensor_list([x], [off]))
    table, scores, grad = torch.zeros(1, 3, device="cuda"), torch.zeros(1, 3, 4, 4, device="cuda"), torch.zeros(1, 3, device="cuda")
    b = qgx.Buckets([-100, 100], [0])
    for off in ((1 << 30) + 1, -(1 << 30) - 1, 1 << 64, (1 << 64) + 1):
        refused(lambda: c.add_position_bias(scores, table, b, q_offset=off))
        refused(lambda: c.position_bias(table, b, 4, 4, q_offset=off))
        refused(lambda: c.position_bias_backward(scores, b, grad, q_offset=off))
    c.close()
