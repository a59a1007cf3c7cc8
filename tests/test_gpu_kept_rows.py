"""Activations kept (qgx_checkpoint) of tensors whose leading dimensions come down to two steps, some of them of one index."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256)
    yield c
    c.close()


@pytest.mark.parametrize("shape,cut", [((2, 3, 1, 6, 8), 4), ((2, 1, 3, 6, 8), 4), ((1, 2, 3, 6, 8), 4), ((2, 3, 1, 1, 6, 8), 4), ((1, 1, 1, 6, 8), 4)])
def test_rows_kept_beside_dimensions_of_one(ctx, shape, cut):
    """Leading dimensions that come down to two steps although one of them has a single index."""
    big = torch.randn(shape, device="cuda")
    x = big[..., :cut, :]
    assert torch.equal(ctx.restore(ctx.checkpoint(x)), ctx.restore(ctx.checkpoint(x.contiguous())))


@pytest.mark.parametrize("shape", [(2, 0, 0, 8), (0, 3, 0, 8), (2, 0, 3, 1, 8), (0, 0, 0, 8)])
def test_nothing_in_many_dimensions(ctx, shape):
    kept = ctx.checkpoint(torch.zeros(shape, device="cuda"), 1)
    assert kept.shape == shape and ctx.restore(kept).shape == shape


def test_rows_of_three_steps_are_refused(ctx):
    from paper_2308_09187_amd import qgx
    x = torch.zeros(2, 4, 1, 6, 10, 8, device="cuda")[:, :3, :, :5, ::2]
    with pytest.raises(qgx.QgxError) as e:
        ctx.checkpoint(x)
    assert e.value.status == qgx.ERR_ARG
