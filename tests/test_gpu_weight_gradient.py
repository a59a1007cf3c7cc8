"""The weight gradient from kept activations (qgx_weight_gradient) against the product in 64 bits.

Whole numbers whose sums stay below 2^24 have to come out exactly, whatever the order.  Other inputs: with u = 2^-24 every product is exact and a sum of n
terms, in any order, is off by at most (n + 8) u of the sum of magnitudes, n = rows times the one, two or three parts of an element of dy."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PARTS = {"f32": 3, "f16": 2, "bf16": 1}
SHAPES = [(1, 1, 1), (1, 7, 3), (2, 32, 1), (5, 33, 129), (63, 64, 64), (64, 128, 128), (65, 100, 127), (128, 129, 130), (200, 257, 5), (300, 5, 300),
          (513, 96, 200), (1000, 260, 70), (4097, 40, 33)]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256)
    yield c
    c.close()


def whole_numbers(seed, K, rows, cols, out, typ, most=8):
    """x in -most .. most with a power of two per row (so that all stays whole), dy alike; sums below rows * (4 most)^2 / 4."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randint(-most, most + 1, (K, rows, cols), generator=g, device="cuda").float()
    x *= torch.exp2(torch.randint(0, 2, (K, rows, 1), generator=g, device="cuda").float())
    dy = torch.randint(-most, most + 1, (K, rows, out), generator=g, device="cuda").to(TYPES[typ])
    return x, dy


def product(x, dy):
    return torch.matmul(x.double().transpose(-1, -2).contiguous(), dy.double())


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("rows,cols,out", SHAPES)
def test_whole_numbers(ctx, rows, cols, out, typ):
    K = 2
    x, dy = whole_numbers(rows, K, rows, cols, out, typ)
    dw, db = torch.full((K, cols, out), 9.0, device="cuda"), torch.full((K, out), 9.0, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw, db)
    assert torch.equal(ctx.restore(ctx.checkpoint(x)), x)
    assert torch.equal(dw.double(), product(x, dy)) and torch.equal(db.double(), dy.double().sum(1))
    dw2 = torch.empty_like(dw)
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw2)
    assert torch.equal(dw, dw2)


@pytest.mark.parametrize("K,rows,cols,out,typ", [(1, 20000, 64, 64, "bf16"), (3, 5000, 300, 520, "bf16"), (1, 9000, 130, 1000, "f16"), (2, 2000, 700, 300, "f32"),
                                                 (8, 64, 1000, 1000, "bf16"), (1, 128, 2050, 2050, "bf16"), (4, 777, 256, 320, "f32")])
def test_whole_numbers_of_larger_layers(ctx, K, rows, cols, out, typ):
    x, dy = whole_numbers(rows, K, rows, cols, out, typ, 4)
    dw, db = torch.empty(K, cols, out, device="cuda"), torch.empty(K, out, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw, db)
    assert torch.equal(dw.double(), product(x, dy)) and torch.equal(db.double(), dy.double().sum(1))


def check(ctx, kept, dy, dw, db, typ):
    x = ctx.restore(kept).double()
    d = dy.double()
    n = dy.shape[-2] * PARTS[typ]
    bound = (n + 8) * U * product(x.abs(), d.abs()) + 2.0 ** -140
    assert bool(((dw.double() - product(x, d)).abs() <= bound).all())
    if db is not None:
        assert bool(((db.double() - d.sum(-2)).abs() <= (dy.shape[-2] + 8) * U * d.abs().sum(-2) + 2.0 ** -140).all())


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("K,rows,cols,out", [(1, 1, 40, 40), (2, 37, 90, 50), (3, 500, 200, 260), (1, 3000, 128, 256)])
def test_numbers(ctx, K, rows, cols, out, typ):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x = torch.randn(K, rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (K, rows, 1), generator=g, device="cuda").float())
    dy = (torch.randn(K, rows, out, generator=g, device="cuda") * 1e-2).to(TYPES[typ])
    kept = ctx.checkpoint(x, 3)
    dw, db = torch.empty(K, cols, out, device="cuda"), torch.empty(K, out, device="cuda")
    ctx.weight_gradient(kept, dy, dw, db)
    check(ctx, kept, dy, dw, db, typ)


def test_all_bits_of_dy_count(ctx):
    """One row: the gradient is a product of two numbers, exact but for its own rounding."""
    dy = torch.randn(1, 1, 300, device="cuda")
    x = torch.tensor([[[1.0, -3.0, 0.0, 127.0]]], device="cuda")
    dw = torch.empty(1, 4, 300, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw)
    want = product(x, dy)
    assert bool(((dw.double() - want).abs() <= 3 * U * want.abs()).all())
    dy = torch.tensor([torch.finfo(torch.float16).max, torch.finfo(torch.float16).tiny, 2.0 ** -24, 1.0009765625], device="cuda").half().view(1, 1, 4)
    dw = torch.empty(1, 4, 4, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw)
    want = product(x, dy)
    assert bool(((dw.double() - want).abs() <= 2 * U * want.abs()).all())


@pytest.mark.parametrize("typ", TYPES)
def test_strides_odd_addresses_and_runs_of_v(ctx, typ):
    K, rows, cols, out = 3, 150, 70, 45
    x, big = whole_numbers(1, K, rows, cols, out + 13, typ)
    dy = big[..., 3:3 + out]
    V = torch.full((K, 11 + cols * out + out + 5), 5.0, device="cuda")
    dw, db = V[:, 11:11 + cols * out].unflatten(1, (cols, out)), V[:, 11 + cols * out:11 + cols * out + out]
    kept = ctx.checkpoint(x)
    ctx.weight_gradient(kept, dy, dw, db)
    assert torch.equal(dw.double(), product(x, dy)) and torch.equal(db.double(), dy.double().sum(1))
    assert bool((V[:, :11] == 5).all()) and bool((V[:, -5:] == 5).all())
    t = big.transpose(0, 1).contiguous().transpose(0, 1)[..., 3:3 + out]              # rows of the workers in turn
    ctx.weight_gradient(kept, t, dw, db)
    assert torch.equal(dw.double(), product(x, dy))
    one = big[:, :1, 3:3 + out].expand(K, rows, out)       # a gradient that is the same for all rows
    ctx.weight_gradient(kept, one, dw, db)
    assert torch.equal(dw.double(), product(x, one)) and torch.equal(db.double(), one.double().sum(1))
    ctx.weight_gradient(ctx.checkpoint(x[0]), dy[0], dw[0], db[0])
    assert torch.equal(dw[0].double(), product(x[0], dy[0]))


@pytest.mark.parametrize("typ", TYPES)
def test_no_numbers(ctx, typ):
    x, dy = whole_numbers(2, 2, 100, 70, 140, typ)
    x[x == 0] = 1.0
    clean = product(x, dy)
    d = dy.clone()
    d[0, 50, 7], d[0, 51, 8], d[1, 99, 130] = math.inf, -math.inf, math.nan
    dw, db = torch.empty(2, 70, 140, device="cuda"), torch.empty(2, 140, device="cuda")
    kept = ctx.checkpoint(x)
    ctx.weight_gradient(kept, d, dw, db)
    want = clean.clone()
    want[0, :, 7], want[0, :, 8], want[1, :, 130] = math.inf * torch.sign(x[0, 50]), -math.inf * torch.sign(x[0, 51]), math.nan
    assert torch.equal(dw.double().nan_to_num(7.0, 1e300, -1e300), want.nan_to_num(7.0, 1e300, -1e300))
    assert float(db[0, 7]) == math.inf and float(db[0, 8]) == -math.inf and math.isnan(float(db[1, 130])) and int(torch.isfinite(db).sum()) == 2 * 140 - 3
    x[1, 3, 40] = math.nan                                 # spoils its block: 32 columns of one worker's gradient
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw, db)
    ctx.poll_error()
    bad = torch.isnan(dw)
    assert bool(bad[1, 32:64].all()) and int(bad.sum()) == 32 * 140
    assert torch.equal(dw[0].double(), clean[0]) and torch.equal(dw[1, :32].double(), clean[1, :32])


def test_unbiased_rounding_gives_the_gradient_on_average(ctx):
    """dW is linear in what was kept: its mean over calls is that of x, off by the mean of rows of errors of at most a step each (Hoeffding)."""
    x, dy = torch.randn(16, 32, device="cuda"), torch.ones(16, 1, device="cuda")
    n, dw, total = 3000, torch.empty(32, 1, device="cuda"), torch.zeros(32, 1, device="cuda", dtype=torch.float64)
    for call in range(n):
        total += ctx.weight_gradient(ctx.checkpoint(x, call), dy, dw).double()
    step = torch.exp2(ctx.checkpoint(x).powers.double() - 127.0)
    spread = float((step ** 2).sum())                      # of the sum's terms' squared ranges
    bound = math.sqrt(math.log(2e12) * spread / (2 * n)) + float(step.sum()) * 2.0 ** -16 + 1e-5
    assert bool(((total / n - x.double().sum(0, keepdim=True).t()).abs() <= bound).all())


def test_against_differences(ctx):
    """y = x W, loss = sum c y: the gradient is the difference of the loss over a step of W, exactly, for a linear layer and whole numbers."""
    x, c = whole_numbers(4, 1, 20, 12, 9, "f32")
    dw = torch.empty(1, 12, 9, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), c, dw)
    W = torch.zeros(12, 9, dtype=torch.float64, device="cuda")
    for i, o in ((0, 0), (3, 8), (11, 4)):
        up = W.clone()
        up[i, o] = 1.0
        loss = (c[0].double() * (x[0].double() @ up)).sum() - (c[0].double() * (x[0].double() @ W)).sum()
        assert float(loss) == float(dw[0, i, o])


@pytest.mark.parametrize("typ", TYPES)
def test_rows_far_apart(ctx, typ):
    """dy's rows 2^24 + 6 elements apart (a step of more than the tiled kernels take), and one column of many."""
    rows, cols, out = 40, 33, 6
    x, d = whole_numbers(6, 1, rows, cols, out, typ)
    dy = torch.empty(rows, (1 << 24) + 6, device="cuda", dtype=TYPES[typ])[:, 5:5 + out]
    dy.copy_(d[0])
    dw, db = torch.empty(cols, out, device="cuda"), torch.empty(out, device="cuda")
    kept = ctx.checkpoint(x[0])
    ctx.weight_gradient(kept, dy, dw, db)
    assert torch.equal(dw.double(), product(x[0], d[0])) and torch.equal(db.double(), d[0].double().sum(0))
    ctx.weight_gradient(kept, dy[:, 2:3], dw[:, :1].contiguous(), db[:1])
    assert float(db[0]) == float(d[0, :, 2].double().sum())
    torch.cuda.empty_cache()


def test_offsets_beyond_32_bits(ctx):
    """More than 2^32 codes, and a dy of more than 2^32 elements, of which only the last rows are no zeros."""
    rows, cols, out, last = (1 << 20) + 77, 4128, 34, 300
    x, d = whole_numbers(7, 1, last, cols, out, "bf16")
    kept = ctx.new_checkpoint((rows, cols))
    kept.codes.fill_(128)
    kept.powers.zero_()
    small = ctx.checkpoint(x[0])
    kept.codes[-last:].copy_(small.codes)
    kept.powers[-last:].copy_(small.powers)
    wide = torch.zeros(rows, 4200, device="cuda", dtype=torch.bfloat16)
    dy = wide[:, 4001:4001 + out]
    dy[-last:].copy_(d[0])
    dw, db = torch.empty(cols, out, device="cuda"), torch.empty(out, device="cuda")
    ctx.weight_gradient(kept, dy, dw, db)
    assert torch.equal(dw.double(), product(x[0], d[0])) and torch.equal(db.double(), d[0].double().sum(0))
    del kept, wide, dy
    torch.cuda.empty_cache()


def test_two_calls_at_once(ctx):
    """Two streams' calls, and two graphs replayed side by side: each has its own memory for the parts' sums."""
    data = [whole_numbers(8 + i, 2, 3000, 96, 200, "bf16") for i in range(2)]
    kept = [ctx.checkpoint(x) for x, _ in data]
    dw = [torch.zeros(2, 96, 200, device="cuda") for _ in data]
    want = [product(x, dy) for x, dy in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        ctx.weight_gradient(kept[i], data[i][1], dw[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a.double(), b) for a, b in zip(dw, want))
    graphs = []
    for i, s in enumerate(streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.weight_gradient(kept[i], data[i][1], dw[i], stream=s)
        graphs.append(g)
    for _ in range(3):
        for t in dw:
            t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.double(), b) for a, b in zip(dw, want))


def test_grids_too_large_are_refused(ctx):
    from paper_2308_09187_amd import qgx
    ask = lambda *a: ctx.lib.qgx_weight_gradient_scratch(ctx._h, *a, ctx._need_ref)  # noqa: E731
    assert ask(2, 65535, 1, 1 << 17, 1 << 13, 1 << 13) == qgx.ERR_ARG
    assert ask(2, 65535, 1, 1 << 10, 1 << 10, 1 << 10) == 0
    assert ask(2, 65535, 1, 1 << 17, 1, 1) == qgx.ERR_ARG


def test_nothing_to_do(ctx):
    dw, db = torch.full((2, 40, 30), 5.0, device="cuda"), torch.full((2, 30), 5.0, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(torch.zeros(2, 0, 40, device="cuda")), torch.zeros(2, 0, 30, device="cuda"), dw, db)
    assert bool((dw == 0).all()) and bool((db == 0).all())
    ctx.weight_gradient(ctx.checkpoint(torch.zeros(0, 3, 40, device="cuda")), torch.zeros(0, 3, 30, device="cuda"), torch.empty(0, 40, 30, device="cuda"))


def test_on_another_stream_and_in_a_graph(ctx):
    x, dy = whole_numbers(5, 2, 3000, 96, 200, "f32")
    kept = ctx.checkpoint(x)
    dw, db = torch.zeros(2, 96, 200, device="cuda"), torch.zeros(2, 200, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.weight_gradient(kept, dy, dw, db, stream=side)
    side.synchronize()
    assert torch.equal(dw.double(), product(x, dy))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.checkpoint(x, out=kept, stream=side)
        ctx.weight_gradient(kept, dy, dw, db, stream=side)
    for _ in range(3):
        x.add_(1.0)
        dy.neg_()
        dw.zero_()
        eager = ctx.weight_gradient(ctx.checkpoint(x), dy, torch.empty_like(dw))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, eager) and torch.equal(dw.double(), product(x, dy)) and torch.equal(db.double(), dy.double().sum(1))


def test_refusals(ctx):
    from paper_2308_09187_amd import qgx
    x, dy = torch.zeros(2, 8, 40, device="cuda"), torch.zeros(2, 8, 30, device="cuda")
    k, dw, db = ctx.checkpoint(x), torch.zeros(2, 40, 30, device="cuda"), torch.zeros(2, 30, device="cuda")

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    refused(lambda: ctx.weight_gradient(k, dy.double(), dw, db))
    refused(lambda: ctx.weight_gradient(k, dy.cpu(), dw, db))
    refused(lambda: ctx.weight_gradient(k, dy[..., ::2], dw[..., :15], db[:, :15]))
    refused(lambda: ctx.weight_gradient(k, dy[:, :7], dw, db))
    refused(lambda: ctx.weight_gradient(k, dy[:1], dw, db))
    refused(lambda: ctx.weight_gradient(k, dy[0], dw[0], db[0]))
    refused(lambda: ctx.weight_gradient(k, dy, dw.bfloat16(), db))
    refused(lambda: ctx.weight_gradient(k, dy, dw[:1], db))
    refused(lambda: ctx.weight_gradient(k, dy, dw.transpose(1, 2), db))
    refused(lambda: ctx.weight_gradient(k, dy, dw, torch.zeros(1, 30, device="cuda").expand(2, 30)))
    refused(lambda: ctx.weight_gradient(k, dy, torch.zeros(1, 40, 30, device="cuda").expand(2, 40, 30)))
    refused(lambda: ctx.weight_gradient(k, dy, None, db))
    refused(lambda: ctx.weight_gradient(k, torch.zeros(2, 8, 0, device="cuda"), torch.zeros(2, 40, 0, device="cuda")))
    h, s = ctx._h, torch.cuda.current_stream().cuda_stream
    lib = ctx.lib
    from ctypes import addressof
    assert lib.qgx_weight_gradient(h, None, 0, 2, 8, 30, dy.data_ptr(), 240, 30, dw.data_ptr(), 1200, None, 0, None, 0, s) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient(h, addressof(k._c), 0, 2, 8, 30, dy.data_ptr(), 240, 30, None, 1200, None, 0, None, 0, s) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient(h, addressof(k._c), 0, 2, 8, 30, dy.data_ptr() + 2, 240, 30, dw.data_ptr(), 1200, None, 0, None, 0, s) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient(h, addressof(k._c), 0, 2, 8, 30, dy.data_ptr(), 1 << 62, 30, dw.data_ptr(), 1200, None, 0, None, 0, s) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient(h, addressof(k._c), 0, 2, 8, 1 << 26, dy.data_ptr(), 240, 30, dw.data_ptr(), 1200, None, 0, None, 0, s) == qgx.ERR_ARG
