"""Group norm with an activation, channels last (qgx_group_norm, qgx_group_norm_backward) against the formulas in 64 bits, the gradients against
differences too.

Bounds, u = 2^-24.  A group's or a channel's sum is made of a thread's places one by one (at most 16, or in parts four turns of four
with a mean's update of three roundings each) and then of the threads' in runs and trees of at most 256 terms more, or of a group wider than that its
entries / 256: S = (320 + places * per / 65536 + parts) u of the sum of magnitudes covers all of them.  mean: S mean|x|; x - mean: that and u |x - mean|; the variance: S and twice
the shift's square over it; rstd half of that and 3 u.  h: relative rstd's error, and the shift times rstd.  z = h w + b: three roundings.  Activations: |silu'| <= 1.1, |silu''|
<= 0.5, the sigmoid good to (6 + 2 |z|) u.  Backward from the given mean and rstd: h by 3 u |h|, or from a kept element by one product and one sum of its code, 2 u (255 scale +
|mean|) rstd; dz by its factor's error; sums as above; dx four more roundings.  Last the type's
own rounding."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
SLOPE = 0.2
# batch, places, channels, groups
SHAPES = [(1, 1, 1, 1), (2, 1, 8, 1), (1, 1, 512, 32), (2, 3, 3, 1), (1, 5, 2, 2), (3, 7, 7, 7), (2, 16, 32, 8), (1, 64, 512, 32), (2, 49, 96, 6), (2, 221, 90, 6),
          (1, 197, 60, 30), (2, 100, 40, 4), (1, 33, 34, 17), (1, 300, 320, 32), (1, 1024, 256, 32), (2, 1000, 24, 1), (1, 4096, 64, 8), (1, 5000, 40, 4), (1, 17, 2100, 3),
          (1, 3, 9001, 1), (1, 20000, 12, 3), (1, 30000, 5, 5), (2, 2049, 130, 13), (1, 9, 600, 300), (1, 700, 66, 33)]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256, seed=77)
    yield c
    c.close()


def make(seed, shape, typ, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * scale
    return (x + torch.randn(shape[-1], generator=g, device="cuda") * scale).to(TYPES[typ])


def params(seed, C):
    g = np.random.default_rng(seed)
    w, b = 1 + 0.3 * g.standard_normal(C), 0.5 * g.standard_normal(C)
    return torch.from_numpy(w).float().cuda(), torch.from_numpy(b).float().cuda()


def host(t):
    return t.double().cpu().numpy()


def act(z, kind):
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if kind == "leaky":
        return np.where(z > 0, z, SLOPE * z), np.where(z > 0, 1.0, SLOPE)
    return z, np.ones_like(z)


def S_of(P, per):
    return (320 + P * per / 65536 + P / 64) * U


def grouped(x, G):
    return x.reshape(x.shape[:-1] + (G, x.shape[-1] // G))


def check_forward(x, G, w, b, eps, kind, y, mean, rstd, typ):
    """x [.., places, channels] numpy; statistics over the places and each group's channels."""
    g = grouped(x, G)
    per = g.shape[-1]
    S = S_of(x.shape[-2], per)
    mu, var = g.mean((-3, -1), keepdims=True), g.var((-3, -1), keepdims=True)
    r = 1 / np.sqrt(var + eps)
    h = (g - mu) * r
    shift = S * np.abs(g).mean((-3, -1), keepdims=True)
    rrel = 0.5 * (S + 2 * shift ** 2 * r ** 2 + 4 * U) + 3 * U
    herr = np.abs(h) * (rrel + 3 * U) + shift * r
    flat = lambda t: np.broadcast_to(t, g.shape).reshape(x.shape)  # noqa: E731
    h, herr = flat(h), flat(herr)
    z = h * w + b
    zerr = herr * np.abs(w) + 2 * U * (np.abs(h * w) + np.abs(b))
    f, _ = act(z, kind)
    err = 1.1 * zerr + (8 + 2 * np.abs(z)) * U * np.abs(f)
    err = err + ROUND[typ] * (np.abs(f) + err) + TINY[typ]
    assert (np.abs(host(y) - f) <= err).all()
    if mean is not None:
        assert (np.abs(host(mean) - mu[..., 0, :, 0]) <= shift[..., 0, :, 0] + U * np.abs(mu[..., 0, :, 0])).all()
        assert (np.abs(host(rstd) / r[..., 0, :, 0] - 1) <= rrel[..., 0, :, 0] + U).all()


def run_forward(ctx, x, G, w, b, kind, typ, eps=1e-5, **kw):
    y, mean, rstd = ctx.group_norm(x, G, w, b, eps, kind, SLOPE, **kw)
    one = np.float64(1)
    check_forward(host(x), G, one if w is None else host(w), 0.0 if b is None else host(b), eps, kind, y, mean, rstd, typ)
    return y, mean, rstd


@pytest.mark.parametrize("kind", ["none", "silu", "leaky"])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("batch,P,C,G", SHAPES)
def test_forward(ctx, batch, P, C, G, typ, kind):
    w, b = params(C, C)
    run_forward(ctx, make(P, (batch, P, C), typ), G, w, b, kind, typ)


@pytest.mark.parametrize("typ", TYPES)
def test_forward_workers_parameters_and_dimensions(ctx, typ):
    x = make(1, (3, 2, 30, 48), typ)
    w, b = params(2, 48)
    for W, B in ((w, b), (None, b), (w, None), (None, None)):
        run_forward(ctx, x, 6, W, B, "silu", typ)
    run_forward(ctx, x[0], 6, w, b, "silu", typ)
    y, m, r = run_forward(ctx, x[0, 0], 6, w, b, "silu", typ)
    assert m.shape == r.shape == (6,)
    y2, m2, r2 = ctx.group_norm(x[0, 0], 6, w, b, 1e-5, "silu", save=False)
    assert torch.equal(y, y2) and m2 is None and r2 is None


@pytest.mark.parametrize("P,C,G", [(30, 45, 5), (3000, 45, 9), (20000, 20, 2), (50, 5, 1)])
@pytest.mark.parametrize("typ", TYPES)
def test_forward_strides_and_in_place(ctx, typ, P, C, G):
    big = make(3, (2, 3, P, C + 9), typ)
    w, b = params(4, C)
    x = big[..., 3:3 + C]
    want, m, r = run_forward(ctx, x.contiguous(), G, w, b, "leaky", typ)
    got = run_forward(ctx, x, G, w, b, "leaky", typ)
    assert all(torch.equal(a, c) for a, c in zip(got, (want, m, r)))
    out = torch.full((3, 2, P, C + 11), 7.0, device="cuda", dtype=TYPES[typ])
    ctx.group_norm(x, G, w, b, 1e-5, "leaky", SLOPE, out=out.transpose(0, 1)[..., 5:5 + C])
    assert torch.equal(out.transpose(0, 1)[..., 5:5 + C], want) and bool((out[..., :5] == 7).all()) and bool((out[..., 5 + C:] == 7).all())
    before = big.clone()
    ctx.group_norm(x, G, w, b, 1e-5, "leaky", SLOPE, out=x)
    assert torch.equal(x, want)
    before[..., 3:3 + C] = want
    assert torch.equal(big, before)
    same = before[:, :1, ..., 3:3 + C].expand(2, 3, P, C)   # read only: samples may coincide
    run_forward(ctx, same, G, w, b, "none", typ)


@pytest.mark.parametrize("P,C,G", [(40, 24, 3), (9000, 24, 3)])
@pytest.mark.parametrize("typ", TYPES)
def test_offsets_constant_groups_and_outliers(ctx, typ, P, C, G):
    w, b = params(5, C)
    x = make(6, (2, P, C), typ)
    x[0] = (x[0].float() * 0.01 + 8.0).to(TYPES[typ])      # far from zero
    x[1, :, :8] = 3.0                                      # a group of one value: y = act(b)
    x[1, 0, 8] = 1000.0                                    # the first element far from all others
    y, mean, rstd = run_forward(ctx, x, G, w, b, "silu", typ)
    z = host(b)[:8] / (1 + np.exp(-host(b)[:8]))
    assert (np.abs(host(y)[1, :, :8] - z) <= (ROUND[typ] + 16 * U) * np.abs(z) + TINY[typ]).all()
    assert float(mean[1, 0]) == 3.0 and abs(float(rstd[1, 0]) * math.sqrt(1e-5) - 1) <= 4 * U


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("P,C,G", [(40, 30, 5), (9000, 30, 5)])
def test_no_numbers_stay_in_their_group(ctx, P, C, G, bad):
    w, b = params(7, C)
    x = make(8, (2, P, C), "bf16")
    dy = make(9, (2, P, C), "bf16")
    clean = ctx.group_norm(x, G, w, b, activation="silu")
    dw, db = torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")
    cdx = ctx.group_norm_backward(dy, x, G, w, b, *clean[1:], "silu", dw=dw, db=db)
    cw = dw.clone()
    x[1, P // 2, 13] = bad                                 # group 2: channels 12 .. 17
    y, m, r = ctx.group_norm(x, G, w, b, activation="silu")
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1, :, 12:18] = False
    assert torch.equal(y[keep], clean[0][keep]) and bool(torch.isnan(y[~keep]).all())
    dx = ctx.group_norm_backward(dy, x, G, w, b, m, r, "silu", dw=dw, db=db)
    assert torch.equal(dx[keep], cdx[keep]) and bool(torch.isnan(dx[~keep]).all())
    ok = torch.ones(C, dtype=torch.bool, device="cuda")
    ok[12:18] = False
    assert torch.equal(dw[ok], cw[ok]) and bool(torch.isnan(dw[~ok]).all())


# -- backward -----------------------------------------------------------------------------------------------------------


def check_backward(x, dy, G, w, b, mean, rstd, kind, dx, dw, db, typ, scale=None):
    """[workers, batch, places, channels] numpy, mean and rstd as the kernel sees them."""
    g = grouped(x, G)
    n = x.shape[-2] * g.shape[-1]
    S = S_of(x.shape[-2], g.shape[-1])
    mu, r = mean[..., None, :, None], rstd[..., None, :, None]
    h = ((g - mu) * r).reshape(x.shape)
    z = h * w + b
    _, d = act(z, kind)
    zerr = 4 * U * (np.abs(h * w) + np.abs(b))
    if scale is not None:
        zerr = zerr + 2 * U * np.abs(w) * ((255 * grouped(scale, G) + np.abs(mu)) * r).reshape(x.shape)
    derr = 0.5 * zerr + (10 + 3 * np.abs(z)) * U * (np.abs(d) + np.abs(z) * 0.25 + 0.25) if kind == "silu" else U * np.abs(d)
    if kind == "leaky":                                    # next to 0 binary32 decides by the header's operations
        xs, f32 = x.astype(np.float32), np.float32
        h32 = ((grouped(xs, G) - mu.astype(f32)) * r.astype(f32)).reshape(x.shape)
        z32 = h32 * np.asarray(w, f32) + np.asarray(b, f32)
        d = np.where(z32 > 0, 1.0, SLOPE)
    dz = dy * d
    dzerr = np.abs(dy) * derr + U * np.abs(dz)
    herr = 3 * U * np.abs(h)
    if scale is not None:
        herr = herr + 2 * U * ((255 * grouped(scale, G) + np.abs(mu)) * r).reshape(x.shape)
    batch = x.shape[1]
    for got, terms, terr in ((dw, dz * h, dzerr * np.abs(h) + np.abs(dz) * herr), (db, dz, dzerr)):
        if got is not None:
            want = terms.sum((1, 2))
            assert (np.abs(host(got) - want) <= (terr + (S + batch * U) * np.abs(terms)).sum((1, 2)) + 2.0 ** -140).all()
    if dx is None:
        return
    k, kerr = dz * w, dzerr * np.abs(w) + U * np.abs(dz * w)
    hg, kg = grouped(h, G), grouped(k, G)

    def mean_of(t):
        return np.broadcast_to(grouped(t, G).sum((-3, -1), keepdims=True) / n, hg.shape).reshape(x.shape)

    m1, m2 = mean_of(k), mean_of(k * h)
    m1err = mean_of(kerr + (S + 4 * U) * np.abs(k))
    m2err = mean_of(kerr * np.abs(h) + np.abs(k) * herr + (S + 4 * U) * np.abs(k * h))
    want = (k - m1 - h * m2)
    err = kerr + m1err + np.abs(h) * m2err + np.abs(m2) * herr + 4 * U * (np.abs(k) + np.abs(m1) + np.abs(h * m2))
    rs = np.broadcast_to(r, hg.shape).reshape(x.shape)
    want, err = want * rs, err * rs + 2 * U * np.abs(want * rs)
    err = err + ROUND[typ] * (np.abs(want) + err) + TINY[typ]
    assert (np.abs(host(dx) - want) <= err).all()


def run_backward(ctx, x, dy, G, w, b, kind, typ, source=None, **kw):
    """x, dy [workers, batch, places, channels]."""
    K, C = x.shape[0], x.shape[-1]
    _, mean, rstd = ctx.group_norm(x, G, w, b, activation=kind, slope=SLOPE)
    dw, db = torch.full((K, C), 9.0, device="cuda"), torch.full((K, C), 9.0, device="cuda")
    dx = ctx.group_norm_backward(dy, x if source is None else source, G, w, b, mean, rstd, kind, SLOPE, dw=dw, db=db, **kw)
    seen = host(x) if source is None else host(ctx.restore(source))
    scale = None if source is None else np.exp2(host(source.powers) - 127.0).repeat(32, -1)[..., :C]
    check_backward(seen, host(dy), G, np.float64(1) if w is None else host(w), np.float64(0) if b is None else host(b), host(mean), host(rstd), kind, dx, dw, db, typ, scale)
    return dx, dw, db


@pytest.mark.parametrize("kind", ["none", "silu", "leaky"])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("batch,P,C,G", SHAPES)
def test_backward(ctx, batch, P, C, G, typ, kind):
    w, b = params(C, C)
    x, dy = make(P, (1, batch, P, C), typ), make(P + 1, (1, batch, P, C), typ, 0.1)
    run_backward(ctx, x, dy, G, w, b, kind, typ)
    run_backward(ctx, x, dy, G, w, b, kind, typ, source=ctx.checkpoint(x, 3))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("K,batch,P,C,G", [(3, 1, 30, 48, 6), (2, 5, 100, 33, 3), (4, 2, 6000, 16, 2), (5, 40, 4, 8, 8)])
def test_backward_workers_and_parameters(ctx, K, batch, P, C, G, typ):
    x, dy = make(1, (K, batch, P, C), typ), make(2, (K, batch, P, C), typ, 0.1)
    w, b = params(3, C)
    for W, B in ((w, b), (None, b), (w, None), (None, None)):
        run_backward(ctx, x, dy, G, W, B, "silu", typ)


@pytest.mark.parametrize("source", ["x", "kept"])
@pytest.mark.parametrize("P,C,G", [(30, 45, 5), (9000, 45, 9)])
@pytest.mark.parametrize("typ", TYPES)
def test_backward_strides_runs_of_v_and_fewer_results(ctx, typ, P, C, G, source):
    K, N = 2, 3
    x, dy = make(4, (K, N, P, C + 7), typ)[..., 2:2 + C], make(5, (K, N, P, C + 4), typ, 0.1)[..., 1:1 + C]
    w, b = params(6, C)
    src = ctx.checkpoint(x, 1) if source == "kept" else None
    dx, dw, db = run_backward(ctx, x, dy, G, w, b, "silu", typ, source=src)
    _, mean, rstd = ctx.group_norm(x, G, w, b, activation="silu")
    V = torch.full((K, 2 * C + 11), 5.0, device="cuda")
    out = torch.full((N, K, P, C + 9), 7.0, device="cuda", dtype=TYPES[typ])
    back = lambda **kw: ctx.group_norm_backward(dy, x if src is None else src, G, w, b, mean, rstd, "silu", **kw)  # noqa: E731
    back(dw=V[:, 3:3 + C], db=V[:, 5 + C:5 + 2 * C], dx=out.transpose(0, 1)[..., 4:4 + C])
    assert torch.equal(out.transpose(0, 1)[..., 4:4 + C], dx) and bool((out[..., :4] == 7).all()) and bool((out[..., 4 + C:] == 7).all())
    assert torch.equal(V[:, 3:3 + C], dw) and torch.equal(V[:, 5 + C:5 + 2 * C], db)
    assert bool((V[:, :3] == 5).all()) and bool((V[:, 3 + C:5 + C] == 5).all()) and bool((V[:, 5 + 2 * C:] == 5).all())
    V.fill_(5.0)
    assert back(dw=V[:, 3:3 + C], need_dx=False) is None and torch.equal(V[:, 3:3 + C], dw)
    back(db=V[:, 1:1 + C], need_dx=False)
    assert torch.equal(V[:, 1:1 + C], db)
    assert torch.equal(back(), dx) and back(need_dx=False) is None


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("K,N,P,C,G", [(2, 3, 64, 40, 4), (1, 2, 7000, 24, 3)])
def test_sums_of_whole_numbers_are_exact(ctx, K, N, P, C, G, typ):
    """mean 0 and rstd 1 given, no activation: dw and db are sums of whole numbers below 2^24."""
    g = torch.Generator(device="cuda")
    g.manual_seed(P)
    x, dy = (torch.randint(-4, 5, (K, N, P, C), generator=g, device="cuda").to(TYPES[typ]) for _ in range(2))
    mean, rstd = torch.zeros(K, N, G, device="cuda"), torch.ones(K, N, G, device="cuda")
    dw, db = torch.empty(K, C, device="cuda"), torch.empty(K, C, device="cuda")
    for src in (x, ctx.checkpoint(x)):
        ctx.group_norm_backward(dy, src, G, None, None, mean, rstd, dw=dw, db=db)
        assert torch.equal(dw.double(), (dy.double() * x.double()).sum((1, 2))) and torch.equal(db.double(), dy.double().sum((1, 2)))


@pytest.mark.parametrize("kind", ["none", "silu", "leaky"])
def test_gradients_against_differences(ctx, kind):
    """Central differences of the forward kernel's binary32 result, sums in 64 bits: step 2^-6, third derivatives below 40 of these sizes
    leave 40 / 6 * 2^-12; the forward's own error, 64 u of 600 terms of size 3, over 2^-5."""
    x, dy = make(11, (1, 2, 10, 12), "f32"), make(12, (1, 2, 10, 12), "f32")
    w, b = params(13, 12)
    if kind == "leaky":                                    # away from the corner: no place within a step's reach of 0
        b += 8.0
    _, m, r = ctx.group_norm(x, 3, w, b, activation=kind, slope=SLOPE)
    dw, db = torch.empty(1, 12, device="cuda"), torch.empty(1, 12, device="cuda")
    dx = ctx.group_norm_backward(dy, x, 3, w, b, m, r, kind, SLOPE, dw=dw, db=db)

    def loss(x, w, b):
        return float((ctx.group_norm(x, 3, w, b, activation=kind, slope=SLOPE, save=False)[0].double() * dy.double()).sum())

    step = 2.0 ** -6
    for t, grad, places in ((x, dx, [(0, 0, 0, 0), (0, 1, 9, 11), (0, 1, 4, 5)]), (w, dw[0], [0, 7]), (b, db[0], [3, 11])):
        for at in places:
            values = []
            for s in (step, -step):
                p = {id(t): t.clone()}
                p[id(t)][at] += s
                values.append(loss(p.get(id(x), x), p.get(id(w), w), p.get(id(b), b)))
            assert abs((values[0] - values[1]) / (2 * step) - float(grad[at])) <= 40 / 6 * step ** 2 + 64 * U * 240 * 3 / (2 * step)


@pytest.mark.parametrize("call", [None, 6])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("K,N,P,C,G", [(2, 2, 64, 64, 8), (1, 3, 50, 96, 32), (2, 1, 77, 45, 5), (1, 1, 9000, 32, 4), (1, 1, 3000, 100, 10), (2, 2, 1024, 256, 32), (1, 2, 5, 3, 1)])
def test_the_input_is_kept_beside(ctx, K, N, P, C, G, typ, call):
    from paper_2308_09187_amd import qgx
    x = make(14, (K, N, P, C + 3), typ)[..., 1:1 + C]
    w, b = params(15, C)
    want = ctx.group_norm(x, G, w, b, activation="silu")
    kept, alone = ctx.new_checkpoint(x.shape), ctx.checkpoint(x, call)
    got = ctx.group_norm(x, G, w, b, activation="silu", keep=kept, call_id=call)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert torch.equal(kept.codes, alone.codes) and torch.equal(kept.powers, alone.powers)
    ctx.group_norm(x, G, w, b, activation="silu", keep=kept, call_id=call, out=x)       # in place: what was there is kept
    assert torch.equal(x, want[0]) and torch.equal(kept.codes, alone.codes) and torch.equal(kept.powers, alone.powers)
    ctx.poll_error()
    x[0, 0, 3, 1] = math.nan
    ctx.group_norm(x, G, w, b, keep=kept, call_id=call)
    assert ctx.poll_error() == qgx.EBIT_NONFINITE
    alone = ctx.checkpoint(x, call)
    assert torch.equal(kept.codes, alone.codes) and torch.equal(kept.powers, alone.powers)
    ctx.poll_error()


def test_offsets_beyond_32_bits(ctx):
    P, C, G = 1 << 16, 40, 5
    big = torch.zeros(3, 1 << 15, P, 1, device="cuda", dtype=torch.bfloat16).view(3, -1)          # 4 GiB a sample
    x = big[:, -P * C:].view(3, P, C)
    x.copy_(make(16, (3, P, C), "bf16"))
    w, b = params(17, C)
    want = ctx.group_norm(x.contiguous(), G, w, b, activation="silu")
    got = ctx.group_norm(x, G, w, b, activation="silu")
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    dy = make(18, (3, P, C), "bf16")
    y = ctx.group_norm_backward(dy, x, G, w, b, *want[1:], "silu")
    assert torch.equal(y, ctx.group_norm_backward(dy, x.contiguous(), G, w, b, *want[1:], "silu"))
    ctx.group_norm_backward(dy, x.contiguous(), G, w, b, *want[1:], "silu", dx=x)
    assert torch.equal(x, y) and float(big[:, :-P * C].abs().max()) == 0
    del big, x
    torch.cuda.empty_cache()


def test_nothing_to_do(ctx):
    w, b = params(1, 8)
    dw, db = torch.full((2, 8), 5.0, device="cuda"), torch.full((2, 8), 5.0, device="cuda")
    for shape in ((2, 0, 4, 8), (2, 3, 0, 8)):
        x = torch.zeros(shape, device="cuda")
        y, m, r = ctx.group_norm(x, 2, w, b)
        assert y.shape == shape
        dw.fill_(5.0)
        db.fill_(5.0)
        dx = ctx.group_norm_backward(x, x.clone(), 2, w, b, m, r, dw=dw, db=db)
        assert dx.shape == shape and bool((dw == 0).all()) and bool((db == 0).all())
    x = torch.zeros(0, 3, 4, 8, device="cuda")
    y, m, r = ctx.group_norm(x, 2, w, b)
    ctx.group_norm_backward(x, x.clone(), 2, w, b, m, r, dw=dw[:0], db=db[:0])


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("P,C,G", [(50, 64, 4), (50, 45, 5), (9000, 64, 4)])
@pytest.mark.parametrize("kind", ["none", "silu", "leaky"])
def test_constant_groups_far_from_zero(ctx, kind, P, C, G, typ):
    """mean * rstd beyond binary32, x - mean 0: z is the bias, dx = rstd (g - mean g), dw 0.  Also of what was kept (3 2^121 is 96 2^116, kept exactly), and
    where places do not fill the threads.  The statistics are given: a forward pass's sum of n of these, 3 n 2^121, is beyond binary32 (2^128) from n = 43 on,
    which the header rules out, so that it has none to offer."""
    x = torch.full((1, 2, P, C), 3 * 2.0 ** 121, device="cuda").to(TYPES[typ])
    w, b = params(2, C)
    mean, rstd = torch.full((1, 2, G), 3 * 2.0 ** 121, device="cuda"), torch.full((1, 2, G), 1e5 ** 0.5, device="cuda")
    _, d = act(host(b), kind)
    dy = make(3, x.shape, typ)
    want = (host(dy) * d).sum((1, 2))
    bound = (S_of(P, 1) + 20 * U) * (np.abs(host(dy)) * np.abs(d)).sum((1, 2))
    for source in (x, ctx.checkpoint(x)):
        dw, db = torch.empty(1, C, device="cuda"), torch.empty(1, C, device="cuda")
        dx = ctx.group_norm_backward(dy, source, G, w, b, mean, rstd, kind, SLOPE, dw=dw, db=db)
        assert bool((dw == 0).all()) and bool(torch.isfinite(dx).all())
        assert (np.abs(host(db) - want) <= bound).all()


def test_two_graphs_at_once(ctx):
    """Two captured steps replayed side by side on two streams: each has its own memory for the parts' sums."""
    P, C, G = 8000, 64, 8
    xs, dys = [make(30 + i, (2, 2, P, C), "bf16") for i in range(2)], [make(40 + i, (2, 2, P, C), "bf16") for i in range(2)]
    w, b = params(50, C)
    want, got, graphs, streams = [], [], [], [torch.cuda.Stream() for _ in xs]

    def step(i, stream=None):
        dw, db = torch.empty(2, C, device="cuda"), torch.empty(2, C, device="cuda")
        y, m, r = ctx.group_norm(xs[i], G, w, b, activation="silu", stream=stream)
        return y, m, r, ctx.group_norm_backward(dys[i], xs[i], G, w, b, m, r, "silu", dw=dw, db=db, stream=stream), dw, db

    for i in range(2):
        want.append(step(i))
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got.append(step(i, s))
        graphs.append(g)
    for _ in range(3):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, want):
            assert all(torch.equal(s, t) for s, t in zip(a, c))
            for t in a:
                t.zero_()


def test_grids_too_large_are_refused(ctx):
    from ctypes import addressof

    from paper_2308_09187_amd import qgx

    def ask(*a):
        shape = qgx._GroupShape(*a)
        return ctx.lib.qgx_group_norm_scratch(ctx._h, addressof(shape), 0, ctx._need_ref)

    assert ask(qgx.DTYPES[torch.float32], 0, 0.0, 1 << 18, 1, 65535, 1, 1 << 20) == qgx.ERR_ARG
    assert ask(qgx.DTYPES[torch.float32], 0, 0.0, 1 << 8, 1, 65535, 1, 1 << 10) == 0


@pytest.mark.parametrize("P", [60, 8000])
def test_on_another_stream_and_in_a_graph(ctx, P):
    K, N, C, G = 2, 2, 64, 8
    x, dy = make(19, (K, N, P, C), "bf16"), make(20, (K, N, P, C), "bf16")
    w, b = params(21, C)
    dw, db, dw2, db2 = (torch.empty(K, C, device="cuda") for _ in range(4))
    want = ctx.group_norm(x, G, w, b, activation="silu")
    wdx = ctx.group_norm_backward(dy, x, G, w, b, *want[1:], "silu", dw=dw, db=db)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ctx.group_norm(x, G, w, b, activation="silu", stream=side)
    gdx = ctx.group_norm_backward(dy, x, G, w, b, *got[1:], "silu", dw=dw2, db=db2, stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got + (gdx, dw2, db2), want + (wdx, dw, db)))
    kept = ctx.new_checkpoint(x.shape)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        y, m, r = ctx.group_norm(x, G, w, b, activation="silu", keep=kept, call_id=4, stream=side)
        dx = ctx.group_norm_backward(dy, kept, G, w, b, m, r, "silu", dw=dw2, db=db2, stream=side)
    for _ in range(3):
        x.mul_(1.25)
        dy.neg_()
        eager = ctx.checkpoint(x, 4)
        ey, em, er = ctx.group_norm(x, G, w, b, activation="silu")
        edx = ctx.group_norm_backward(dy, eager, G, w, b, em, er, "silu", dw=dw, db=db)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((y, m, r, dx, dw2, db2), (ey, em, er, edx, dw, db)))


def test_refusals(ctx):
    from paper_2308_09187_amd import qgx
    x = torch.zeros(2, 3, 4, 8, device="cuda")
    w, m, p = torch.ones(8, device="cuda"), torch.zeros(2, 3, 2, device="cuda"), torch.zeros(2, 8, device="cuda")
    y = x.clone()

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    refused(lambda: ctx.group_norm(x.double(), 2, w, w))
    refused(lambda: ctx.group_norm(x.cpu(), 2, w, w))
    refused(lambda: ctx.group_norm(x[..., ::2], 2, w[:4], w[:4]))
    refused(lambda: ctx.group_norm(x, 3, w, w))
    refused(lambda: ctx.group_norm(x, 0, w, w))
    refused(lambda: ctx.group_norm(x, -2, w, w))
    refused(lambda: ctx.group_norm(x, 2, w[:7], w))
    refused(lambda: ctx.group_norm(x, 2, w.bfloat16(), w))
    refused(lambda: ctx.group_norm(x, 2, w, w, eps=-1.0))
    refused(lambda: ctx.group_norm(x, 2, w, w, eps=math.nan))
    refused(lambda: ctx.group_norm(x, 2, w, w, activation="relu6"))
    refused(lambda: ctx.group_norm(x, 2, w, w, activation="leaky", slope=math.inf))
    refused(lambda: ctx.group_norm(x, 2, w, w, activation="leaky", slope=math.nan))
    refused(lambda: ctx.group_norm(x, 2, w, w, out=x[:1].expand(2, 3, 4, 8)))
    refused(lambda: ctx.group_norm(x, 2, w, w, out=x.bfloat16()))
    refused(lambda: ctx.group_norm(x, 2, w, w, keep=ctx.new_checkpoint((2, 3, 4, 9))))
    refused(lambda: ctx.group_norm(x, 2, w, w, keep=ctx.new_checkpoint((6, 4, 8))))
    refused(lambda: ctx.group_norm(x, 2, w, w, keep=ctx.new_checkpoint(x.shape), call_id=-1))
    refused(lambda: ctx.group_norm(torch.zeros(8, device="cuda"), 2, w, w))
    refused(lambda: ctx.group_norm(torch.zeros(1, 2, 3, 4, 8, device="cuda"), 2, w, w))
    refused(lambda: ctx.group_norm(torch.zeros(2, 3, 0, device="cuda"), 1))
    back = lambda dy=y, src=x, g=2, W=w, B=w, M=m, R=m, **kw: ctx.group_norm_backward(dy, src, g, W, B, M, R, **kw)  # noqa: E731
    refused(lambda: back(dx=x))
    refused(lambda: back(dx=y))
    refused(lambda: back(dy=y.bfloat16()))
    refused(lambda: back(src=x[:1]))
    refused(lambda: back(src=ctx.new_checkpoint((2, 3, 4, 9))))
    refused(lambda: back(M=m[:1]))
    refused(lambda: back(M=None))
    refused(lambda: back(R=m.half()))
    refused(lambda: back(g=5))
    refused(lambda: back(dw=p[:1]))
    refused(lambda: back(dw=p.bfloat16()))
    refused(lambda: back(dw=p, db=torch.zeros(2, 9, device="cuda")[:, :8]))
    refused(lambda: back(dw=torch.zeros(1, 8, device="cuda").expand(2, 8)))
