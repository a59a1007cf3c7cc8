"""The weight gradient (qgx_weight_gradient) where one column of dy, or rows far apart, take the kernel without pairs of columns, over many steps of rows and
many parts.

Whole numbers whose sums stay below 2^24 have to come out exactly, whatever the order."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256)
    yield c
    c.close()


def whole_numbers(seed, K, rows, cols, out, typ, most=8):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randint(-most, most + 1, (K, rows, cols), generator=g, device="cuda").float()
    x *= torch.exp2(torch.randint(0, 2, (K, rows, 1), generator=g, device="cuda").float())
    return x, torch.randint(-most, most + 1, (K, rows, out), generator=g, device="cuda").to(TYPES[typ])


def product(x, dy):
    return torch.matmul(x.double().transpose(-1, -2).contiguous(), dy.double())


def parts_of(ctx, typ, K, rows, cols, out, step):
    from paper_2308_09187_amd import qgx
    assert ctx.lib.qgx_weight_gradient_scratch(ctx._h, qgx.DTYPES[TYPES[typ]], K, rows, cols, out, step, ctx._need_ref) == 0
    return max(1, ctx._need_bytes.value // (4 * K * (cols + 1) * out))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("K,rows,cols", [(1, 1, 1), (2, 63, 40), (2, 64, 128), (2, 65, 129), (1, 128, 300), (3, 129, 33), (2, 193, 64), (1, 1000, 5), (2, 4097, 260), (1, 20000, 96),
                                         (4, 3001, 1000)])
def test_one_column(ctx, K, rows, cols, typ):
    x, dy = whole_numbers(rows, K, rows, cols, 1, typ)
    dw, db = torch.full((K, cols, 1), 9.0, device="cuda"), torch.full((K, 1), 9.0, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(x), dy, dw, db)
    assert torch.equal(dw.double(), product(x, dy)) and torch.equal(db.double(), dy.double().sum(1))
    alone = torch.empty_like(dw)
    ctx.weight_gradient(ctx.checkpoint(x), dy, alone)
    assert torch.equal(alone, dw)


def test_one_column_in_one_part_in_few_and_in_many(ctx):
    """(The rows above reach every join: none, by one thread and by sixteen.)"""
    parts = [parts_of(ctx, "bf16", K, rows, cols, 1, 1) for K, rows, cols in ((2, 193, 64), (1, 1000, 5), (1, 20000, 96), (4, 3001, 1000))]
    assert min(parts) <= 2 and any(1 < p <= 16 for p in parts) and max(parts) > 16


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("rows,cols,out", [(70, 33, 6), (200, 140, 3)])
def test_rows_far_apart(ctx, rows, cols, out, typ):
    """dy's rows 2^24 + 6 elements apart, more than a step of them, and one column of those."""
    x, d = whole_numbers(6, 1, rows, cols, out, typ)
    dy = torch.empty(rows, (1 << 24) + 6, device="cuda", dtype=TYPES[typ])[:, 5:5 + out]
    dy.copy_(d[0])
    kept = ctx.checkpoint(x[0])
    for at, n in ((0, out), (2, 1)):
        dw, db = torch.full((cols, n), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        ctx.weight_gradient(kept, dy[:, at:at + n], dw, db)
        assert torch.equal(dw.double(), product(x[0], d[0][:, at:at + n])) and torch.equal(db.double(), d[0][:, at:at + n].double().sum(0))
    del dy
    torch.cuda.empty_cache()
