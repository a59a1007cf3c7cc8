"""Group norm (qgx_group_norm) of batches without places: the statistics are no numbers."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256, seed=78)
    yield c
    c.close()


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("shape,G", [((2, 3, 0, 8), 2), ((5, 0, 64), 8), ((0, 6), 3), ((40, 50, 0, 96), 32), ((2, 0, 4, 8), 2)])
def test_statistics_of_no_places(ctx, shape, G, typ):
    """The mean of nothing is no number, nor is its spread; nothing else is written."""
    x = torch.zeros(shape, device="cuda", dtype=TYPES[typ])
    kept = ctx.new_checkpoint(x.shape)
    used = [torch.full((2,) + tuple(shape[:-2]) + (G,), 5.0, device="cuda") for _ in range(3)]       # (memory that held numbers)
    del used
    y, mean, rstd = ctx.group_norm(x, G, keep=kept, call_id=1)
    assert y.shape == x.shape and mean.shape == rstd.shape == x.shape[:-2] + (G,)
    assert bool(torch.isnan(mean).all()) and bool(torch.isnan(rstd).all()) and ctx.poll_error() == 0
    assert ctx.group_norm(x, G, save=False)[1:] == (None, None)


def test_statistics_of_no_places_on_another_stream_and_in_a_graph(ctx):
    x = torch.zeros(2, 3, 0, 8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, mean, rstd = ctx.group_norm(x, 4, stream=side)
    side.synchronize()
    assert bool(torch.isnan(mean).all()) and bool(torch.isnan(rstd).all())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        y, mean, rstd = ctx.group_norm(x, 4, stream=side)
    for _ in range(3):
        mean.zero_()
        rstd.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert bool(torch.isnan(mean).all()) and bool(torch.isnan(rstd).all())
