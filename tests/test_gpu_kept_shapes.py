"""Kept activations in the shapes that their uses have: weight gradients from [workers, batch, places, channels], and other leading dimensions of the same rows.

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


@pytest.mark.parametrize("typ", TYPES)
def test_kept_in_their_natural_shape(ctx, typ):
    """[workers, batch, places, channels], as a group norm keeps its input: the rows of a worker are its places."""
    K, N, P, C, out = 2, 3, 50, 40, 30
    x, dy = whole_numbers(4, K, N * P, C, out, typ)
    kept = ctx.checkpoint(x.view(K, N, P, C))
    want, bias = product(x, dy), dy.double().sum(1)

    def check(kept, dy, *lead):
        dw, db = torch.full(lead + (C, out), 9.0, device="cuda"), torch.full(lead + (out,), 9.0, device="cuda")
        ctx.weight_gradient(kept, dy, dw, db)
        assert torch.equal(dw.double(), want if lead else want[0]) and torch.equal(db.double(), bias if lead else bias[0])

    check(kept, dy.view(K, N, P, out), K)
    wide = torch.full((K, N * P, out + 5), 7.0, device="cuda", dtype=TYPES[typ])
    wide[..., 2:2 + out] = dy
    check(kept, wide[..., 2:2 + out].view(K, N, P, out), K)
    check(ctx.checkpoint(x.view(K, N, 5, 10, C)), wide[..., 2:2 + out].view(K, N, 5, 10, out), K)
    turned = dy.view(K, N * P, out).transpose(0, 1).contiguous().transpose(0, 1)
    check(kept, turned.view(K, N, P, out), K)
    # the same memory in another shape
    check(kept.view((K, N * P, C)), dy, K)
    assert kept.view((K, N * P, C)).codes.data_ptr() == kept.codes.data_ptr() and torch.equal(ctx.restore(kept.view((K * N, P, C))).view(K, N * P, C), x)
    one = ctx.checkpoint(x[0].view(N, P, C), tensor=3)     # of a model without workers
    check(one.view((N * P, C)), dy[0])
    assert one.view((N * P, C)).tensor == 3
    split = ctx.checkpoint(x.view(K, N, P, C))
    check(type(split)(split.codes, split.powers, C).view((K, N * P, C)), dy, K)


def test_shapes_that_do_not_go_together_are_refused(ctx):
    from paper_2308_09187_amd import qgx
    kept = ctx.checkpoint(torch.zeros(2, 3, 5, 40, device="cuda"))
    dw = torch.zeros(2, 40, 30, device="cuda")

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    refused(lambda: ctx.weight_gradient(kept, torch.zeros(2, 3, 7, 30, device="cuda")[:, :, :5], dw))         # rows of no one step
    refused(lambda: ctx.weight_gradient(kept, torch.zeros(3, 2, 5, 30, device="cuda"), dw))
    refused(lambda: ctx.weight_gradient(kept, torch.zeros(2, 15, 30, device="cuda"), dw))
    refused(lambda: ctx.weight_gradient(kept, torch.zeros(2, 3, 5, 30, device="cuda"), dw[:1]))
    refused(lambda: kept.view((2, 15, 39)))
    refused(lambda: kept.view((2, 14, 40)))
    refused(lambda: kept.view(()))


def test_nothing_in_more_dimensions(ctx):
    dw, db = torch.full((2, 40, 30), 5.0, device="cuda"), torch.full((2, 30), 5.0, device="cuda")
    ctx.weight_gradient(ctx.checkpoint(torch.zeros(2, 0, 4, 40, device="cuda")), torch.zeros(2, 0, 4, 30, device="cuda"), dw, db)
    assert bool((dw == 0).all()) and bool((db == 0).all())
