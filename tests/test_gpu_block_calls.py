"""Calls of the block's operators with tensors that look alike share what the binding has worked out: another step, type or place must not be taken for the
one before, a refused call leaves nothing, and more shapes than are remembered are no matter.  Everything is compared with a fresh context's call, bit for bit."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pair():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = [m.Context(1024, 1, 256, seed=4) for _ in range(2)]
    yield c
    for x in c:
        x.close()


def fresh(ctx):
    ctx._calls.clear()
    return ctx


def refused(f):
    from paper_2308_09187_amd import qgx
    with pytest.raises(qgx.QgxError) as e:
        f()
    assert e.value.status == qgx.ERR_ARG


def test_group_norm(pair):
    ctx, other = pair
    big = torch.randn(4, 6, 40, 64, device="cuda")
    w, b = torch.randn(32, device="cuda"), torch.randn(32, device="cuda")
    for x in (big[:2, :3, :, :32], big[2:, 3:, :, 32:], big[:2, :3, :, :32].contiguous(), big.transpose(0, 1)[:2, :3, :, :32], big[:2, :3, :, :32].half()):
        for kind in ("silu", "none"):
            got, want = ctx.group_norm(x, 4, w, b, activation=kind), fresh(other).group_norm(x.clone(), 4, w, b, activation=kind)
            assert all(torch.equal(s, t) for s, t in zip(got, want))
            dx = ctx.group_norm_backward(x, x, 4, w, b, *got[1:], kind)
            assert torch.equal(dx, fresh(other).group_norm_backward(x.clone(), x.clone(), 4, w, b, *got[1:], kind))
        refused(lambda: ctx.group_norm(x, 4, w[:16], b))
        refused(lambda: ctx.group_norm(x, 5, w, b))
        refused(lambda: ctx.group_norm(x, 4, w, b, keep=ctx.new_checkpoint(x.shape[1:])))
        refused(lambda: ctx.group_norm_backward(x, x, 4, w, b, got[1][:1], got[2]))


def test_weight_gradient(pair):
    ctx, other = pair
    big = torch.randint(-4, 5, (4, 50, 80), device="cuda").float()
    kept = [ctx.checkpoint(torch.randint(-4, 5, (2, 50, 40), device="cuda").float()) for _ in range(2)]
    V = torch.zeros(2, 40 * 30 + 30, device="cuda")
    runs = V[:, :1200].unflatten(1, (40, 30)), V[:, 1200:]
    for k in kept:
        for dy in (big[:2, :, :30], big[2:, :, 7:37], big[::2, :, :30], big[:2, :, :30].contiguous(), big[:2, :, :30].bfloat16()):
            dw, db = torch.empty(2, 40, 30, device="cuda"), torch.empty(2, 30, device="cuda")
            ctx.weight_gradient(k, dy, dw, db)
            ctx.weight_gradient(k, dy, *runs)
            want = torch.matmul(ctx.restore(k).transpose(1, 2).double(), dy.double())
            assert torch.equal(dw.double(), want) and torch.equal(runs[0].double(), want) and torch.equal(runs[1], db)
            refused(lambda: ctx.weight_gradient(k, dy, dw[:, :39], db))
            refused(lambda: ctx.weight_gradient(k, dy, dw.half(), db))
            refused(lambda: ctx.weight_gradient(k, dy[:, :49], dw, db))


def test_rotary(pair):
    from paper_2308_09187_amd import qgx
    ctx, other = pair
    big = torch.randn(3, 5, 7, 4, 40, device="cuda")
    p = torch.randint(0, 99, (2, 3, 5, 7), dtype=torch.int32, device="cuda")
    rotations = [qgx.Rotary.by_base((5, 5)), qgx.Rotary.by_base((3, 4), neighbours=True)]
    for x in (big[..., :20], big[..., 20:], big[..., :20].contiguous(), big[..., :20].transpose(2, 3).contiguous().transpose(2, 3), big[..., :20].bfloat16()):
        for r in rotations:
            for pos in (p, p.flip(3).contiguous(), p[:, 0, 0]):
                got, want = ctx.rotary(x, r, pos), fresh(other).rotary(x.clone(), r, pos)
                y = x.clone()
                assert torch.equal(got, want) and torch.equal(ctx.rotary(y, r, pos, out=y), want)
            refused(lambda: ctx.rotary(x, r, p.long()))
            refused(lambda: ctx.rotary(x, r, p[:1]))
            refused(lambda: ctx.rotary(x, r, p, out=x[:1]))


def test_more_shapes_than_are_remembered(pair):
    ctx, _ = pair
    for n in range(1, 600):
        x = torch.ones(n, 8, device="cuda")
        assert ctx.group_norm(x, 2, eps=1.0)[0].shape == x.shape
    assert len(ctx._calls) <= 512 and ctx.poll_error() == 0
    x = torch.randn(9, 8, device="cuda")
    assert torch.allclose(ctx.group_norm(x, 2)[0], torch.nn.functional.group_norm(x.t().unsqueeze(0).contiguous(), 2)[0].t(), atol=1e-5)
