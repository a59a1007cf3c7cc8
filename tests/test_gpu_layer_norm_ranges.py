"""Layer norm's backward pass on rows whose spread is far from 1: the formulas' values are ordinary numbers, while rstd^2, or a gradient
times a deviation, lies outside binary32.  Bounds: those of test_gpu_layer_norm.py (errors relative to what is multiplied, whatever the
exponents, as long as no product of the formulas leaves the normal numbers, which the inputs see to)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_layer_norm import check_backward, ctx, host, put, rnd  # noqa: E402, F401

pytestmark = pytest.mark.gpu
# a form for each: shorter than a piece, 4 to 64 threads to a row, 256 by one, two and four pieces, 1024 by two and four, the long ones
COLS = [3, 20, 64, 100, 250, 513, 1001, 2049, 4100, 9000, 16384, 20000]


def gradients(ctx, x, dy, w, mean, rstd, parts):  # noqa: F811
    K, _, cols = x.shape
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw if parts else None, db=db if parts else None)
    return host(dx), host(dw) if parts else None, host(db) if parts else None


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_small_variance_without_epsilon(ctx, cols, typ):  # noqa: F811
    """The forward pass of rows of 1e-20 with eps = 0, and its own mean and rstd (about 1e20) into the backward pass."""
    K, rows = 2, 5
    x, dy = put(1e-20 * rnd((1, cols), K, rows, cols), typ), put(0.1 * rnd((2, cols), K, rows, cols), typ)
    w = put(1 + 0.3 * rnd(3, cols), "f32")
    y, mean, rstd = ctx.layer_norm(x, w, None, 0.0)
    assert bool(torch.isfinite(y).all()) and bool((rstd > 1e19).all()) and bool(torch.isfinite(rstd).all())
    for parts in (True, False):
        dx, dw, db = gradients(ctx, x, dy, w, mean, rstd, parts)
        check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, dx, dw, db)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("spread,size", [(1e-30, 1e-20), (1e25, 1e15)])
@pytest.mark.parametrize("cols", COLS)
def test_gradients_times_deviations_outside_binary32(ctx, cols, spread, size, typ):  # noqa: F811
    K, rows = 2, 5
    x, dy = put(spread * rnd((4, cols), K, rows, cols), typ), put(size * rnd((5, cols), K, rows, cols), typ)
    w = put(1 + 0.3 * rnd(6, cols), "f32")
    xh = host(x)
    mean = put(xh.mean(-1), "f32")
    rstd = put(1 / xh.std(-1), "f32")
    dx, dw, db = gradients(ctx, x, dy, w, mean, rstd, True)
    check_backward(host(dy), xh, host(w), host(mean), host(rstd), typ, dx, dw, db)
