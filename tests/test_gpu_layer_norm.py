"""Layer norm and its backward pass (qgx_layer_norm, qgx_layer_norm_backward) against the formulas in 64 bits, and the
gradients against differences.

Bounds, with u = 2^-24.  A row's sums are made of runs of at most 64 terms (or, beyond 32768 columns, cols / 1024) added one by
one and joined in ten steps: relative to the sum of magnitudes they are off by at most S = (74 + cols / 1024) u.  Forward: the mean is off by
S mean|x|, x - mean by that and 2 u |x|, the variance by S and twice the shift's square (second order), rstd by as much and 4 u; y adds three roundings.
Backward, from the given mean and rstd: h is off by 3 u |h| + u |x| rstd, g by u |g|, the two means by S + 6 u of theirs; dx adds four roundings.
The columns' sums take every row once, in any order: (rows + 16) u of the sum of magnitudes.  Last the rounding to the type."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
COLS = [1, 2, 3, 5, 8, 17, 31, 32, 33, 64, 100, 127, 128, 255, 256, 257, 511, 512, 513, 1000, 1001, 1024, 1025, 2047, 2048, 2049, 4096,
        4097, 6000, 8192, 8193, 16384, 16385, 32768, 32769, 50001]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256)
    yield c
    c.close()


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def put(x, typ):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(TYPES[typ])


def host(t):
    return t.double().cpu().numpy()


def sum_bound(cols):
    return (74 + cols / 1024) * U


def check_forward(x, w, b, eps, typ, y, mean, rstd):
    """x, w, b as the kernel sees them, in 64 bits."""
    cols = x.shape[-1]
    S = sum_bound(cols)
    mu = x.mean(-1, keepdims=True)
    var = ((x - mu) ** 2).mean(-1, keepdims=True)
    r = 1 / np.sqrt(var + eps)
    h = (x - mu) * r
    exact = h * w + b
    shift = S * np.abs(x).mean(-1, keepdims=True) + 2 * U * np.abs(x).max(-1, keepdims=True)
    vrel = S + (shift ** 2 + 2 * shift * U) * r ** 2 * 2
    rrel = vrel + 4 * U
    # where the spread of a row is no more than the error of its mean, the bound says nothing: such rows are tested apart
    bound = np.abs(w) * (r * (shift + 2 * U * np.abs(x)) + np.abs(h) * (rrel + 3 * U)) + 2 * U * (np.abs(h * w) + np.abs(exact))
    bound = 1.01 * bound + ROUND[typ] * (np.abs(exact) + bound) + TINY[typ]
    assert (np.abs(y - exact) <= bound).all(), (np.abs(y - exact) / bound).max()
    if mean is not None:
        assert (np.abs(mean - mu[..., 0]) <= shift[..., 0]).all()
        assert (np.abs(rstd - r[..., 0]) <= 1.01 * (rrel * r)[..., 0]).all()


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_forward(ctx, cols, typ):
    K, rows = 2, 5
    x = put(2 * rnd(cols, K, rows, cols) + rnd(1, K, rows, 1), typ)
    w, b = put(1 + 0.3 * rnd(2, cols), "f32"), put(0.5 * rnd(3, cols), "f32")
    y, mean, rstd = ctx.layer_norm(x, w, b, 1e-5)
    check_forward(host(x), host(w), host(b), float(np.float32(1e-5)), typ, host(y), host(mean), host(rstd))
    y2, m2, _ = ctx.layer_norm(x, w, b, 1e-5, save=False)
    assert m2 is None and torch.equal(y, y2)
    for a, c in ((w, None), (None, b), (None, None)):
        z, _, _ = ctx.layer_norm(x, a, c, 1e-5)
        check_forward(host(x), 1.0 if a is None else host(a), 0.0 if c is None else host(c), float(np.float32(1e-5)), typ, host(z), None, None)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("rows", [1, 2, 3, 63, 257, 1030])
def test_forward_rows_strides_and_in_place(ctx, rows, typ):
    cols = 199
    wide = put(rnd(rows, 3, rows, 2 * cols + 3), typ)
    keep = wide.clone()
    x = wide[:, :, 3:3 + cols]                                  # odd step between rows, odd start
    w, b = put(rnd(2, 2 * cols), "f32")[1:1 + cols], put(rnd(3, cols + 1), "f32")[1:]
    y, mean, rstd = ctx.layer_norm(x, w, b, 1e-5)
    assert y.is_contiguous()
    check_forward(host(x), host(w), host(b), float(np.float32(1e-5)), typ, host(y), host(mean), host(rstd))
    t, _, _ = ctx.layer_norm(x.transpose(0, 1), w, b, 1e-5)     # the workers in the middle
    assert torch.equal(t.transpose(0, 1), y)
    ctx.layer_norm(x, w, b, 1e-5, out=x)
    assert torch.equal(x, y)
    assert torch.equal(wide[:, :, :3], keep[:, :, :3]) and torch.equal(wide[:, :, 3 + cols:], keep[:, :, 3 + cols:])


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("cols", [3, 1001, 16390, 32769, 50001])
def test_in_place_of_any_length(ctx, cols, typ):
    x, w, b = put(rnd((5, cols), 2, 3, cols + 3), typ), put(rnd(6, cols), "f32"), put(rnd(7, cols), "f32")
    view = x[..., 2:2 + cols]
    keep, want = x.clone(), ctx.layer_norm(view, w, b)[0]
    ctx.layer_norm(view, w, b, out=view)
    assert torch.equal(view, want) and torch.equal(x[..., :2], keep[..., :2]) and torch.equal(x[..., 2 + cols:], keep[..., 2 + cols:])


def test_one_token(ctx):
    x = put(rnd(1, 1000), "bf16")
    w, b = put(rnd(2, 1000), "f32"), put(rnd(3, 1000), "f32")
    y, mean, rstd = ctx.layer_norm(x, w, b)
    assert y.shape == x.shape and mean.shape == ()
    check_forward(host(x), host(w), host(b), float(np.float32(1e-5)), "bf16", host(y), host(mean), host(rstd))


def test_constant_rows_large_offsets_and_no_numbers(ctx):
    cols = 300
    x = np.zeros((6, cols))
    x[0] = 7.0                                                  # no spread: y = bias, rstd = 1 / sqrt(eps)
    x[1] = 1e4 + rnd(1, cols)                                   # a mean far from 0: the second pass keeps the spread
    x[2] = rnd(2, cols); x[2, 17] = np.nan
    x[3] = rnd(3, cols); x[3, 299] = np.inf
    x[4] = 1e-30 * rnd(4, cols)
    x[5] = rnd(5, cols)
    t = put(x, "f32")
    b = put(rnd(6, cols), "f32")
    y, mean, rstd = ctx.layer_norm(t, None, b, 1e-5)
    yh, bh = host(y), host(b)
    assert np.array_equal(yh[0], bh) and abs(host(rstd)[0] - 1e-5 ** -0.5) < 1e-4
    x64 = host(t)
    exact = (x64[1] - x64[1].mean()) / np.sqrt(x64[1].var() + 1e-5) + bh
    assert np.abs(yh[1] - exact).max() < 1e-2                   # 1e4 times 80 u, over a spread of 1
    assert np.isnan(yh[2]).all() and np.isnan(yh[3]).all()
    check_forward(x64[4:], 1.0, bh, float(np.float32(1e-5)), "f32", yh[4:], host(mean)[4:], host(rstd)[4:])


def plain_backward(dy, x, w, mean, rstd):
    h = (x - mean[..., None]) * rstd[..., None]
    g = dy * w
    dx = rstd[..., None] * (g - g.mean(-1, keepdims=True) - h * (g * h).mean(-1, keepdims=True))
    return dx, (dy * h).sum(-2), dy.sum(-2), h, g


def check_backward(dy, x, w, mean, rstd, typ, dx, dw, db):
    S, rows = sum_bound(x.shape[-1]), x.shape[-2]
    ex, ew, eb, h, g = plain_backward(dy, x, w, mean, rstd)
    r, ag, ah = rstd[..., None], np.abs(g), np.abs(h)
    dh = 3 * U * ah + 2 * U * np.abs(x) * r
    m1, m2 = ag.mean(-1, keepdims=True), (ag * ah).mean(-1, keepdims=True)
    e2 = (S + 8 * U) * m2 + (ag * dh).mean(-1, keepdims=True)
    if dx is not None:
        bound = r * (4 * U * (ag + m1 + ah * m2) + (S + 6 * U) * m1 + ah * e2 + dh * m2) * 1.05
        bound = bound + ROUND[typ] * (np.abs(ex) + bound) + TINY[typ]
        assert (np.abs(dx - ex) <= bound).all(), (np.abs(dx - ex) / bound).max()
    if dw is not None:
        bw = (rows + 16) * U * (np.abs(dy) * ah).sum(-2) + (np.abs(dy) * dh).sum(-2) * 1.05 + TINY["f32"]
        assert (np.abs(dw - ew) <= bw).all(), (np.abs(dw - ew) / bw).max()
    if db is not None:
        bb = (rows + 16) * U * np.abs(dy).sum(-2) + TINY["f32"]
        assert (np.abs(db - eb) <= bb).all(), (np.abs(db - eb) / bb).max()


def back_inputs(K, rows, cols, typ, seed=0):
    x = put(2 * rnd((seed, 1, cols), K, rows, cols) + rnd((seed, 2), K, rows, 1), typ)
    dy = put(0.1 * rnd((seed, 3, cols), K, rows, cols), typ)
    w = put(1 + 0.3 * rnd((seed, 4), cols), "f32")
    xh = host(x)
    mean = xh.mean(-1)
    rstd = 1 / np.sqrt(((xh - mean[..., None]) ** 2).mean(-1) + 1e-5)
    return x, dy, w, put(mean, "f32"), put(rstd, "f32")


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_backward(ctx, cols, typ):
    K, rows, d = 2, 7, cols + 13
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, typ)
    V = torch.full((K, 2 * d), 9.0, device="cuda")
    dw, db = V[:, 5:5 + cols], V[:, d + 5:d + 5 + cols]
    dx = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw, db=db)
    check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, host(dx), host(dw), host(db))
    assert bool((V[:, :5] == 9).all()) and bool((V[:, 5 + cols:d + 5] == 9).all()) and bool((V[:, d + 5 + cols:] == 9).all())


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("K,rows,cols", [(1, 1, 96), (1, 1, 5000), (3, 2, 700), (2, 64, 40), (1, 1000, 260), (4, 333, 129), (1, 4097, 24),
                                         (8, 50, 2050), (2, 1500, 1024), (1, 700, 9000), (2, 40, 33000)])
def test_backward_rows(ctx, K, rows, cols, typ):
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, typ, seed=1)
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw, db=db)
    check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, host(dx), host(dw), host(db))
    # again: the same bits
    dw2, db2 = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx2 = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw2, db=db2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("want", ["dx", "dw", "db", "dw db", "none", "dx db", "dx no weight"])
def test_backward_parts(ctx, want):
    K, rows, cols = 2, 130, 301
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, "bf16", seed=2)
    w = None if "no weight" in want else w
    dw = torch.empty(K, cols, device="cuda") if "dw" in want else None
    db = torch.empty(K, cols, device="cuda") if "db" in want else None
    dx = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw, db=db, need_dx="dx" in want)
    assert (dx is not None) == ("dx" in want)
    check_backward(host(dy), host(x), 1.0 if w is None else host(w), host(mean), host(rstd), "bf16", None if dx is None else host(dx),
                   None if dw is None else host(dw), None if db is None else host(db))


@pytest.mark.parametrize("typ", list(TYPES))
def test_backward_strides(ctx, typ):
    K, rows, cols = 3, 37, 211
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, typ, seed=3)
    xs, gs, out = (torch.zeros(K, rows, cols + pad, device="cuda", dtype=TYPES[typ]) for pad in (3, 7, 5))
    xs[..., 1:1 + cols] = x
    gs[..., 5:5 + cols] = dy
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx = ctx.layer_norm_backward(gs[..., 5:5 + cols], xs[..., 1:1 + cols], w, mean, rstd, dw=dw, db=db, dx=out[..., 2:2 + cols])
    check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, host(dx), host(dw), host(db))
    assert bool((out[..., :2] == 0).all()) and bool((out[..., 2 + cols:] == 0).all())
    one = dy[:, :1].expand(K, rows, cols)                       # a gradient broadcast over the rows
    dx = ctx.layer_norm_backward(one, x, w, mean, rstd, dw=dw, db=db)
    check_backward(host(one), host(x), host(w), host(mean), host(rstd), typ, host(dx), host(dw), host(db))


def test_a_row_of_no_numbers_stays_in_its_row_and_worker(ctx):
    K, rows, cols = 2, 40, 500
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, "f32", seed=4)
    dy[1, 7, 3] = float("nan")
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx = host(ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=dw, db=db))
    assert np.isnan(dx[1, 7]).all()
    dx[1, 7] = 0
    assert np.isfinite(dx).all() and np.isfinite(host(dw)[0]).all()
    bad = np.isnan(host(db)[1])
    assert bad[3] and bad.sum() == 1


def test_gradients_against_differences(ctx):
    """Differences of sum(y * c) in 64 bits, at the kernel's own mean and rstd."""
    rows, cols, eps, step = 4, 37, 1e-5, 1e-6
    x, w, b, c = (np.float32(a).astype(np.float64) for a in (rnd(1, rows, cols), 1 + 0.2 * rnd(2, cols), rnd(3, cols), rnd(4, rows, cols)))

    def loss(x, w, b):
        h = (x - x.mean(-1, keepdims=True)) / np.sqrt(x.var(-1, keepdims=True) + eps)
        return ((h * w + b) * c).sum()

    tx, tw, tb = put(x, "f32"), put(w, "f32"), put(b, "f32")
    _, mean, rstd = ctx.layer_norm(tx, tw, tb, eps)
    dw, db = torch.empty(1, cols, device="cuda"), torch.empty(1, cols, device="cuda")
    dx = host(ctx.layer_norm_backward(put(c, "f32"), tx, tw, mean, rstd, dw=dw, db=db))
    args = [x, w, b]
    for at, got in ((0, dx), (1, host(dw)[0]), (2, host(db)[0])):
        num = np.zeros_like(args[at])
        for i in np.ndindex(*num.shape):
            d = np.zeros_like(num)
            d[i] = step
            num[i] = (loss(*[a + d if j == at else a for j, a in enumerate(args)]) - loss(*[a - d if j == at else a for j, a in enumerate(args)])) / (2 * step)
        # second-order differences: 1e-12 times third derivatives, cancellation 1e-16 |loss| / 1e-6; binary32: 1e-5 of the largest
        assert np.abs(num - got).max() <= 2e-5 * max(1.0, np.abs(num).max())


def test_offsets_beyond_32_bits(ctx):
    K, rows, cols, far = 2, 3, 1001, (1 << 32) + 24
    memory = torch.empty(far + (1 << 20), device="cuda", dtype=torch.bfloat16)
    view = lambda at: memory.as_strided((K, rows, cols), (far, 1024, 1), at)
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, "bf16", seed=9)
    xs, gs, ys = view(0), view(100001), view(200002)
    xs.copy_(x)
    gs.copy_(dy)
    y, m, r = ctx.layer_norm(xs, w, w, out=ys)
    y2, m2, r2 = ctx.layer_norm(x, w, w)
    assert torch.equal(ys, y2) and torch.equal(m, m2) and torch.equal(r, r2)
    check_forward(host(x), host(w), host(w), 1e-5, "bf16", host(ys), host(m), host(r))
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    dx = ctx.layer_norm_backward(gs, xs, w, mean, rstd, dw=dw, db=db, dx=view(300003))
    check_backward(host(dy), host(x), host(w), host(mean), host(rstd), "bf16", host(dx), host(dw), host(db))


def test_nothing_to_do(ctx):
    x = torch.empty(2, 0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, mean, rstd = ctx.layer_norm(x, w, w)
    assert y.shape == (2, 0, 64) and mean.shape == (2, 0)
    dw, db = torch.ones(2, 64, device="cuda"), torch.ones(2, 64, device="cuda")
    ctx.layer_norm_backward(x, x, w, mean, rstd, dw=dw, db=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_on_another_stream_and_in_a_graph(ctx):
    K, rows, cols = 2, 300, 640
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, "bf16", seed=5)
    b = torch.zeros(cols, device="cuda")
    dw, db = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    y, m, r = ctx.layer_norm(x, w, b)
    dx = ctx.layer_norm_backward(dy, x, w, m, r, dw=dw, db=db)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    dw2, db2 = torch.empty(K, cols, device="cuda"), torch.empty(K, cols, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    y2, m2, r2 = ctx.layer_norm(x, w, b, stream=s)
    dx2 = ctx.layer_norm_backward(dy, x, w, m2, r2, dw=dw2, db=db2, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y3, m3, r3 = ctx.layer_norm(x, w, b)
        dx3 = ctx.layer_norm_backward(dy, x, w, m3, r3, dw=dw2, db=db2)
    for i in range(3):
        x.normal_()
        dy.normal_()
        g.replay()
        torch.cuda.synchronize()
        y, m, r = ctx.layer_norm(x, w, b)
        dx = ctx.layer_norm_backward(dy, x, w, m, r, dw=dw, db=db)
        assert torch.equal(y, y3) and torch.equal(dx, dx3) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_refusals(ctx):
    from paper_2308_09187_amd import qgx
    x = torch.zeros(2, 3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    m = torch.zeros(2, 3, device="cuda")
    p = torch.zeros(2, 64, device="cuda")

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    refused(lambda: ctx.layer_norm(x.double(), w, w))
    refused(lambda: ctx.layer_norm(x.cpu(), w, w))
    refused(lambda: ctx.layer_norm(x[..., ::2], w[:32], w[:32]))
    refused(lambda: ctx.layer_norm(x, w[:63], w))
    refused(lambda: ctx.layer_norm(x, w.bfloat16(), w))
    refused(lambda: ctx.layer_norm(x, w, w, eps=-1.0))
    refused(lambda: ctx.layer_norm(x, w, w, eps=float("nan")))
    refused(lambda: ctx.layer_norm(x, w, w, out=x[:1].expand(2, 3, 64)))           # rows that overlap
    refused(lambda: ctx.layer_norm(x, w, w, out=x.bfloat16()))
    refused(lambda: ctx.layer_norm(torch.zeros(2, 2, 3, 64, device="cuda"), w, w))
    refused(lambda: ctx.layer_norm(torch.zeros(2, 3, 0, device="cuda"), None, None))
    refused(lambda: ctx.layer_norm_backward(x, x.clone(), w, m, m, dx=x))
    refused(lambda: ctx.layer_norm_backward(x.clone(), x, w, m, m, dx=x))
    refused(lambda: ctx.layer_norm_backward(x.bfloat16(), x, w, m, m))
    refused(lambda: ctx.layer_norm_backward(x.clone(), x, w, m[:1], m))
    refused(lambda: ctx.layer_norm_backward(x.clone(), x, w, m, m, dw=p[:1]))
    refused(lambda: ctx.layer_norm_backward(x.clone(), x, w, m, m, dw=p.bfloat16()))
    refused(lambda: ctx.layer_norm_backward(x.clone(), x, w, m, m, dw=p, db=torch.zeros(2, 100, device="cuda")[:, :64]))
