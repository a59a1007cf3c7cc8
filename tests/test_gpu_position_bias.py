"""Learned relative position bias by buckets (qgx_position_bias, qgx_position_bias_backward) against the definition in 64 bits.

Bounds: a biased score is one binary32 addition, 2^-24 of it, and the rounding to its type.  A gradient adds n terms in some order:
n 2^-24 of the sum of magnitudes at most (n: the places that take the row), and its own rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
FAR = 1 << 30
# name: (bounds, rows, table rows)
BUCKETS = {
    "causal": ([-FAR, -63, -31, -15, -7, -6, -5, -4, -3, -2, -1, 0, 1], [11, 10, 9, 8, 7, 6, 5, 4, 3, 2, 1, 0], 12),
    "both": ([-FAR, -40, -20, -10, -5, -2, -1, 0, 1, 2, 3, 6, 11, 21, FAR], [6, 5, 4, 3, 2, 1, 0, 7, 8, 9, 10, 11, 12, 13], 16),
    "window": ([-17, -9, -4, 0, 1], [3, 2, 1, 0], 4),
    "shared": ([-FAR, -8, 9, FAR], [1, 0, 1], 3),              # one row for both sides, one row for none
    "ahead": ([100, FAR], [0], 1),                             # most queries see nothing
    "every": (list(range(-64, 65)), list(range(128)), 128),    # the most intervals there are, one delta each
    "one": ([-FAR, FAR], [0], 1),
}


@pytest.fixture(scope="module")
def qgx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    m.load()
    return m


@pytest.fixture(scope="module")
def ctx(qgx):
    c = qgx.Context(1024, 1, 256)
    yield c
    c.close()


def put(x, typ):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(TYPES[typ])


def host(t):
    return t.double().cpu().numpy()


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def rows_of(name, q, k, p):
    """[q, k]: the row that (i, j) takes, -1 where masked."""
    bounds, rows, _ = BUCKETS[name]
    delta = np.arange(k)[None, :] - np.arange(q)[:, None] - p
    at = np.searchsorted(np.array(bounds), delta, side="right") - 1
    out = np.full((q, k), -1)
    ok = (at >= 0) & (at < len(rows))
    out[ok] = np.array(rows)[at[ok]]
    return out


def check_out(got, scores, table, row, typ):
    """row [.., q, k] beside scores [.., heads, q, k]."""
    bias = np.where(row[..., None] >= 0, table[np.maximum(row, 0)], -np.inf)       # [.., q, k, heads]
    bias = np.moveaxis(bias, -1, -3)
    seen = np.broadcast_to(np.isfinite(bias), got.shape)
    with np.errstate(invalid="ignore"):
        exact = np.broadcast_to(bias if scores is None else scores + bias, got.shape)
    assert (got[~seen] == -np.inf).all()
    g, e = got[seen], exact[seen]
    same = (g == e) | (np.isnan(g) & np.isnan(e))
    with np.errstate(invalid="ignore"):
        assert (same | (np.abs(g - e) <= (U + ROUND[typ]) * 1.001 * np.abs(e) + TINY[typ])).all()


SHAPES = [(1, 1), (1, 2), (2, 1), (1, 65), (7, 9), (8, 8), (16, 24), (33, 31), (64, 64), (65, 129), (130, 66), (197, 197), (3, 1000), (1000, 3), (256, 512)]


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", list(BUCKETS))
@pytest.mark.parametrize("q,k", SHAPES)
def test_forward(ctx, qgx, q, k, name, typ):
    N, heads = 2, 3
    bounds, rows, R = BUCKETS[name]
    b = qgx.Buckets(bounds, rows)
    table, scores = put(rnd(1, R, heads), "f32"), put(2 * rnd((q, k), N, heads, q, k), typ)
    for p in (0, k - q, 5, -300):
        row = rows_of(name, q, k, p)
        out = ctx.add_position_bias(scores, table, b, q_offset=p)
        check_out(host(out), host(scores), host(table), row, typ)
        alone = ctx.position_bias(table, b, q, k, dtype=TYPES[typ], q_offset=p)
        assert alone.shape == (heads, q, k)
        check_out(host(alone), None, host(table), row, typ)
    twin = scores.clone()
    assert ctx.add_position_bias(twin, table, b, q_offset=-300, out=twin) is twin and torch.equal(twin, out)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", ["causal", "window", "both"])
@pytest.mark.parametrize("q,k", [(1, 1), (1, 77), (1, 4099), (2, 300), (5, 64)])
def test_tokens_of_sequences_of_different_lengths(ctx, qgx, q, k, name, typ):
    N, heads = 6, 5
    bounds, rows, R = BUCKETS[name]
    table, scores = put(rnd(1, R, heads), "f32"), put(rnd(2, N, heads, q, k), typ)
    pos = np.array([0, k - 1, k // 2, k + 100, -3, min(7, k - 1)])
    scores[0, :, :, 1:] = float("nan")                        # beyond a sequence's end anything may lie
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    out = ctx.add_position_bias(scores, table, qgx.Buckets(bounds, rows), q_offset=1, positions=p)
    check_out(host(out), host(scores), host(table), np.stack([rows_of(name, q, k, 1 + x) for x in pos]), typ)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", ["causal", "both", "every"])
@pytest.mark.parametrize("q,k", [(1, 1100), (3, 1100), (1, 2600), (1, 1024)])
def test_tokens_of_many_sequences(ctx, qgx, q, k, name, typ):
    N, heads = 350, 8                                         # enough that a wave takes several pieces
    bounds, rows, R = BUCKETS[name]
    b = qgx.Buckets(bounds, rows)
    table, scores = put(rnd(1, R, heads), "f32"), put(rnd(2, N, heads, q, k), typ)
    pos = np.random.default_rng(3).integers(-5, k + 70, N)
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    out = ctx.add_position_bias(scores, table, b, positions=p)
    check_out(host(out), host(scores), host(table), np.stack([rows_of(name, q, k, x) for x in pos]), typ)
    ctx.add_position_bias(scores, table, b, positions=p, out=scores)
    assert torch.equal(scores, out)


@pytest.mark.parametrize("typ", list(TYPES))
def test_masked_and_special_scores(ctx, qgx, typ):
    heads, n = 2, 40
    low = float(torch.finfo(TYPES[typ]).min)
    scores = put(rnd(1, 1, heads, n, n), typ)
    scores[..., 3] = float("-inf")
    scores[..., 5] = low
    scores[..., 7] = float("nan")
    scores[..., 9] = float("inf")
    bounds, rows, R = BUCKETS["causal"]
    table = put(rnd(2, R, heads), "f32")
    out = host(ctx.add_position_bias(scores, table, qgx.Buckets(bounds, rows)))
    check_out(out, host(scores), host(table), rows_of("causal", n, n, 0), typ)
    seen = rows_of("causal", n, n, 0) >= 0
    assert (out[0, :, :, 3] == -np.inf).all()
    assert np.isnan(out[0, 0, :, 7][seen[:, 7]]).all() and (out[0, 0, :, 7][~seen[:, 7]] == -np.inf).all()


def test_positions_beyond_the_range_count_as_its_end(ctx, qgx):
    bounds, rows, R = BUCKETS["both"]
    table, scores = put(rnd(1, R, 1), "f32"), put(rnd(2, 3, 1, 1, 50), "f32")
    p = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30], dtype=torch.int32, device="cuda")
    for off in (0, FAR, -FAR):
        out = ctx.add_position_bias(scores, table, qgx.Buckets(bounds, rows), q_offset=off, positions=p)
        pos = np.clip(off + p.cpu().numpy().astype(np.int64), -FAR, FAR)
        check_out(host(out), host(scores), host(table), np.stack([rows_of("both", 1, 50, x) for x in pos]), "f32")


def expect_grad(ds, name, heads, p):
    """[K, R, heads], its bound's sum of magnitudes and number of terms."""
    R = BUCKETS[name][2]
    K, N, H, q, k = ds.shape
    row = rows_of(name, q, k, p)
    out, mag, count = np.zeros((K, R, heads)), np.zeros((K, R, heads)), np.zeros(R)
    for r in range(R):
        at = row == r
        out[:, r] = ds[..., at].sum((1, 3))
        mag[:, r] = np.abs(ds[..., at]).sum((1, 3))
        count[r] = N * at.sum()
    return out, mag, count


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("name", list(BUCKETS))
@pytest.mark.parametrize("q,k", SHAPES)
def test_gradient(ctx, qgx, q, k, name, typ):
    K, N, heads = 2, 3, 3
    bounds, rows, R = BUCKETS[name]
    b = qgx.Buckets(bounds, rows)
    ds = put(0.1 + rnd((q, k), K, N, heads, q, k), typ)
    V = torch.full((K, R * heads + 11), 9.0, device="cuda")
    dt = V[:, 5:5 + R * heads].unflatten(1, (R, heads))
    for p in (0, k - q, 37):
        clean = ds.clone()
        masked = torch.from_numpy(rows_of(name, q, k, p) < 0).cuda()
        clean[..., masked] = float("nan")                     # masked places are not read
        ctx.position_bias_backward(clean, b, dt, q_offset=p)
        exact, mag, count = expect_grad(host(ds), name, heads, p)
        got = host(dt)
        assert (np.abs(got - exact) <= (count[None, :, None] + 2) * U * mag + TINY["f32"]).all()
        assert bool((V[:, :5] == 9).all()) and bool((V[:, 5 + R * heads:] == 9).all())
        again = torch.empty(K, R, heads, device="cuda")
        ctx.position_bias_backward(clean, b, again, q_offset=p)
        assert torch.equal(again, dt)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("K,N,heads,q,k", [(1, 1, 1, 2000, 2000), (3, 9, 2, 130, 140), (1, 40, 5, 31, 17), (1, 2, 1, 1, 20000), (1, 1, 2, 9000, 9)])
def test_gradient_of_larger_batches(ctx, qgx, K, N, heads, q, k, typ):
    for name in ("causal", "both"):
        bounds, rows, R = BUCKETS[name]
        ds = put(0.1 + rnd(1, K, N, heads, q, k), typ)
        dt = torch.empty(K, R, heads, device="cuda")
        ctx.position_bias_backward(ds, qgx.Buckets(bounds, rows), dt)
        exact, mag, count = expect_grad(host(ds), name, heads, 0)
        assert (np.abs(host(dt) - exact) <= (count[None, :, None] + 2) * U * mag + TINY["f32"]).all()


@pytest.mark.parametrize("typ", list(TYPES))
def test_strides(ctx, qgx, typ):
    K, N, heads, q, k = 2, 3, 4, 45, 53
    bounds, rows, R = BUCKETS["both"]
    b = qgx.Buckets(bounds, rows)
    wide = put(rnd(1, N, q, K, heads, k + 9), typ)
    x = wide.permute(2, 0, 3, 1, 4)[..., 3:3 + k]              # [K, N, heads, q, k], heads and queries the other way round in memory
    table = put(rnd(2, R, heads), "f32")
    out = ctx.add_position_bias(x, table, b)
    assert out.is_contiguous()
    check_out(host(out), host(x), host(table), rows_of("both", q, k, 0), typ)
    keep = wide.clone()
    dt = torch.empty(K, R, heads, device="cuda")
    ctx.position_bias_backward(x, b, dt)
    exact, mag, count = expect_grad(host(x), "both", heads, 0)
    assert (np.abs(host(dt) - exact) <= (count[None, :, None] + 2) * U * mag + TINY["f32"]).all()
    ctx.add_position_bias(x, table, b, out=x)
    assert torch.equal(x, out) and torch.equal(wide[..., :3], keep[..., :3]) and torch.equal(wide[..., 3 + k:], keep[..., 3 + k:])
    one = put(rnd(3, 1, N, 1, q, k), typ).expand(K, N, heads, q, k)     # a gradient broadcast over workers and heads
    ctx.position_bias_backward(one, b, dt)
    exact, mag, count = expect_grad(host(one), "both", heads, 0)
    assert (np.abs(host(dt) - exact) <= (count[None, :, None] + 2) * U * mag + TINY["f32"]).all()


def test_gradient_against_differences(ctx, qgx):
    """Differences of sum(softmax(scores + bias) * c) in 64 bits; the kernel gets that loss' gradient of the scores."""
    heads, n, step = 2, 21, 1e-6
    bounds, rows, R = BUCKETS["causal"]
    row = rows_of("causal", n, n, 0)
    table, scores, c = rnd(1, R, heads), rnd(2, heads, n, n), rnd(3, heads, n, n)

    def probs(table):
        z = scores + np.moveaxis(np.where(row[..., None] >= 0, table[np.maximum(row, 0)], -np.inf), -1, 0)
        e = np.exp(z - z.max(-1, keepdims=True))
        return e / e.sum(-1, keepdims=True)

    P = probs(table)
    ds = P * (c - (P * c).sum(-1, keepdims=True))
    dt = torch.empty(R, heads, device="cuda")
    ctx.position_bias_backward(put(ds[None], "f32"), qgx.Buckets(bounds, rows), dt)
    num = np.zeros((R, heads))
    for i in np.ndindex(R, heads):
        d = np.zeros_like(table)
        d[i] = step
        num[i] = ((probs(table + d) * c).sum() - (probs(table - d) * c).sum()) / (2 * step)
    # differences: 1e-16 |loss| / 1e-6 and 1e-12 third derivatives; binary32 gradients of at most 1 in sums of up to 21 x 21
    assert np.abs(num - host(dt)).max() <= 1e-5 * max(1.0, np.abs(num).max())


@pytest.mark.parametrize("q,k", [(1, 1500), (40, 45), (9, 5)])
def test_offsets_beyond_32_bits(ctx, qgx, q, k):
    N, heads, far = 2, 3, (1 << 32) + 24
    bounds, rows, R = BUCKETS["causal"]
    b = qgx.Buckets(bounds, rows)
    memory = torch.empty(far + (1 << 20), device="cuda", dtype=torch.bfloat16)
    view = lambda at: memory.as_strided((N, heads, q, k), (far, q * k + 11, k, 1), at)
    x, table = put(rnd(1, N, heads, q, k), "bf16"), put(rnd(2, R, heads), "f32")
    xs = view(0).copy_(x)
    out = ctx.add_position_bias(xs, table, b, q_offset=k - q, out=view(300001))
    check_out(host(out), host(x), host(table), rows_of("causal", q, k, k - q), "bf16")
    dt = torch.empty(R, heads, device="cuda")
    ctx.position_bias_backward(xs, b, dt, q_offset=k - q)
    exact, mag, count = expect_grad(host(x)[None], "causal", heads, k - q)
    assert (np.abs(host(dt) - exact[0]) <= (count[:, None] + 2) * U * mag[0] + TINY["f32"]).all()


def test_nothing_to_do(ctx, qgx):
    b = qgx.Buckets(*BUCKETS["causal"][:2])
    table = torch.zeros(12, 3, device="cuda")
    for shape in ((0, 3, 4, 4), (2, 3, 0, 4), (2, 3, 4, 0)):
        x = torch.empty(shape, device="cuda")
        assert ctx.add_position_bias(x, table, b).shape == shape
        dt = torch.ones(12, 3, device="cuda")
        ctx.position_bias_backward(x, b, dt)
        assert bool((dt == 0).all())


def test_on_another_stream_and_in_a_graph(ctx, qgx):
    b = qgx.Buckets(*BUCKETS["both"][:2])
    table = torch.randn(16, 4, device="cuda")
    x = torch.randn(2, 3, 4, 100, 120, device="cuda")
    dt, dt2 = torch.empty(2, 16, 4, device="cuda"), torch.empty(2, 16, 4, device="cuda")
    out = ctx.add_position_bias(x, table, b)
    ctx.position_bias_backward(x, b, dt)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out2 = ctx.add_position_bias(x, table, b, stream=s)
    ctx.position_bias_backward(x, b, dt2, stream=s)
    s.synchronize()
    assert torch.equal(out, out2) and torch.equal(dt, dt2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out3 = ctx.add_position_bias(x, table, b)
        ctx.position_bias_backward(x, b, dt2)
    for i in range(3):
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        out = ctx.add_position_bias(x, table, b)
        ctx.position_bias_backward(x, b, dt)
        assert torch.equal(out, out3) and torch.equal(dt, dt2)


def test_refusals(ctx, qgx):
    good = qgx.Buckets(*BUCKETS["causal"][:2])
    table = torch.zeros(12, 3, device="cuda")
    x = torch.zeros(2, 3, 8, 8, device="cuda")
    dt = torch.zeros(12, 3, device="cuda")

    def refused(f, status=qgx.ERR_ARG):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == status and str(e.value)

    refused(lambda: qgx.Buckets([0, 1], [0, 1]))
    for bounds, rows in (([0, 0], [0]), ([1, 0], [0]), ([0], []), ([0, 1], [12]), (list(range(130)), [0] * 129)):
        refused(lambda: ctx.add_position_bias(x, table, qgx.Buckets(bounds, rows)))
        refused(lambda: ctx.position_bias_backward(x, qgx.Buckets(bounds, rows), dt))
    refused(lambda: ctx.add_position_bias(x, table[:, :2], good))
    refused(lambda: ctx.add_position_bias(x, table.double(), good))
    refused(lambda: ctx.add_position_bias(x.double(), table, good))
    refused(lambda: ctx.add_position_bias(x.cpu(), table, good))
    refused(lambda: ctx.add_position_bias(x.transpose(2, 3), table, good))
    refused(lambda: ctx.add_position_bias(x, table, good, out=x.bfloat16()))
    refused(lambda: ctx.add_position_bias(x, table, good, out=torch.zeros(2, 3, 8, 9, device="cuda")))
    refused(lambda: ctx.add_position_bias(x, table, good, out=torch.zeros(2, 3, 1, 8, device="cuda").expand(2, 3, 8, 8)))
    refused(lambda: ctx.add_position_bias(x, table, good, q_offset=(1 << 30) + 1))
    refused(lambda: ctx.add_position_bias(x, table, good, positions=torch.zeros(3, dtype=torch.int32, device="cuda")))
    refused(lambda: ctx.add_position_bias(x, table, good, positions=torch.zeros(2, dtype=torch.int64, device="cuda")))
    refused(lambda: ctx.position_bias_backward(x, good, dt[:, :2]))
    refused(lambda: ctx.position_bias_backward(x, good, dt.bfloat16()))
    refused(lambda: ctx.position_bias_backward(x[None], good, dt))
    refused(lambda: ctx.position_bias_backward(x.expand(2, 2, 3, 8, 8), good, torch.zeros(3, 12, 3, device="cuda")))
