"""The position bias and its gradient where bounds and offsets lie at the ends of their ranges, and the gradient of large squares, exactly:
its inputs are 0, 1, 2 or 3 and no table row takes more than 2^22 of them, so that every partial sum is a whole number below 2^24 and the result
has to be equal, in whatever order it was summed."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_position_bias import BUCKETS, TYPES, ctx, host, put, qgx  # noqa: E402, F401

pytestmark = pytest.mark.gpu
FAR, LOW, HIGH = 1 << 30, -(1 << 31), (1 << 31) - 1
# (bounds, rows, table rows, q_offset)
RANGES = {
    "starts at the end": ([-FAR, 0, HIGH - 1, HIGH], [0, 1, 2], 4, 0),
    "many start far off": ([LOW, -3, 1, 3 << 29, HIGH - 2, HIGH - 1, HIGH], [0, 1, 2, 3, 4, 3], 5, 7),
    "ends at the start": ([LOW, LOW + 1, 0, 5], [2, 1, 0], 3, -FAR),
    "ends at the start, near": ([LOW, LOW + 1, LOW + 2, 0, 5], [2, 1, 3, 0], 4, 0),
    "offset at its end": ([-FAR - 900, -FAR - 20, -FAR, -FAR + 7, FAR, 3 << 29, HIGH], [0, 1, 2, 3, 4, 5], 6, FAR),
    "offset at its start": ([LOW, -3 << 29, -FAR, FAR - 9, FAR, FAR + 30, FAR + 800], [0, 1, 2, 3, 4, 5], 6, -FAR),
    "bound at the offset": ([0, FAR, HIGH], [1, 0], 2, FAR),
    "far bound at the offset": ([-FAR, 3 << 29, HIGH], [1, 0], 2, FAR),
    "everything": ([LOW, HIGH], [0], 1, 0),
}


def rows_of(bounds, rows, q, k, p):
    delta = np.arange(k, dtype=np.int64)[None, :] - np.arange(q, dtype=np.int64)[:, None] - p
    at = np.searchsorted(np.array(bounds, np.int64), delta, side="right") - 1
    out = np.full((q, k), -1)
    ok = (at >= 0) & (at < len(rows))
    out[ok] = np.array(rows)[at[ok]]
    return out


def check_gradient(ctx, qgx, bounds, rows, R, p, K, N, heads, q, k, typ):  # noqa: F811
    ds = np.random.default_rng((q, k)).integers(0, 4, (K, N, heads, q, k)).astype(np.float32)
    row = rows_of(bounds, rows, q, k, p)
    t = put(ds, typ)
    t[..., torch.from_numpy(row < 0).cuda()] = float("nan")
    dt = torch.full((K, R, heads), -1.0, device="cuda")
    ctx.position_bias_backward(t, qgx.Buckets(bounds, rows), dt, q_offset=p)
    ds = ds.sum(1, dtype=np.float64)                           # [K, heads, q, k]
    for r in range(R):
        at = row == r
        assert N * at.sum() <= 1 << 22
        assert np.array_equal(host(dt)[:, r], ds[..., at].sum(-1)), r


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", list(RANGES))
@pytest.mark.parametrize("q,k", [(2000, 2000), (197, 197), (1, 3000), (1, 40), (300, 1100), (9, 3)])
def test_gradient_of_far_ranges(ctx, qgx, q, k, name, typ):  # noqa: F811
    bounds, rows, R, p = RANGES[name]
    check_gradient(ctx, qgx, bounds, rows, R, p, 1, 1, 2, q, k, typ)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", list(RANGES))
@pytest.mark.parametrize("q,k", [(130, 197), (1, 3000), (3, 40), (9, 3)])
def test_forward_of_far_ranges(ctx, qgx, q, k, name, typ):  # noqa: F811
    bounds, rows, R, p = RANGES[name]
    heads = 2
    table, scores = put(np.arange(R * heads).reshape(R, heads) + 1, "f32"), put(np.random.default_rng(q).integers(-9, 9, (1, heads, q, k)), typ)
    out = ctx.add_position_bias(scores, table, qgx.Buckets(bounds, rows), q_offset=p)
    row = rows_of(bounds, rows, q, k, p)
    bias = np.moveaxis(np.where(row[..., None] >= 0, host(table)[np.maximum(row, 0)], -np.inf), -1, 0)
    assert np.array_equal(host(out), host(scores) + bias)      # (small whole numbers: exact in every type)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", list(BUCKETS))
@pytest.mark.parametrize("K,N,heads,q,k", [(1, 1, 1, 2000, 2000), (2, 3, 3, 197, 197), (3, 9, 2, 130, 140), (1, 40, 5, 31, 17), (1, 2, 1, 1, 20000),
                                           (1, 1, 2, 9000, 9), (1, 1, 1, 700, 5000), (2, 2, 2, 1019, 1019), (1, 6, 1, 5, 900), (1, 3, 2, 1000, 3)])
def test_gradient_exactly(ctx, qgx, K, N, heads, q, k, name, typ):  # noqa: F811
    bounds, rows, R = BUCKETS[name]
    check_gradient(ctx, qgx, bounds, rows, R, 0, K, N, heads, q, k, typ)
