"""Clipping into a V that lies between its tensors in memory, or between the workers' parts of one: the same norms and the same V, bit for bit,
as a V elsewhere.  And a V that shares any of their memory, which may not take the form for a V apart from it.

That the sums have one order shows only where the order decides a rounding.  With m = 2^24 + 1, which lies half-way between two numbers of
binary32, m^2 = (2^24)^2 + 4096^2 + 4096^2 + 1 is exact in binary64, and its last place is 2^(48 - 52) = 2^-4.  Elements of 2^-3 after these
four leave the sum at m^2 if they are added one by one (2^-6 each, below half a place), and the norm then rounds to 2^24; four of them added up
first are a whole place, and with seven places or more the norm, whose own are 2^-28, is above m by 7 2^-4 / 2^25 and rounds to 2^24 + 2."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PIECE = 4096


@pytest.fixture(scope="module")
def qgx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    m.load()
    return m


def half_way(K, n, cut):
    """Four elements in every 4096 of the two tensors."""
    x = np.zeros((K, n), np.float32)
    for at in (*range(0, cut, PIECE), *range(cut, n, PIECE)):
        x[:, at:at + 4] = 0.125
    x[:, :4] = 2.0 ** 24, 4096, 4096, 1
    x[1:] *= 2.0                                               # (another worker, the same of twice the size)
    return x


def random(K, n, cut=0):
    return np.random.default_rng(n).standard_normal((K, n)).astype(np.float32)


def clipped(qgx, ctx, tensors, offsets, V, limit, kind):
    got = ctx.clip_gradients(ctx.tensor_list(tensors, offsets), limit, norm=qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF, out=V)
    return got.cpu().numpy(), V.cpu().numpy()


@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("make", [half_way, random])
@pytest.mark.parametrize("cut", [5 * PIECE, 7 * PIECE + 13])
@pytest.mark.parametrize("n", [10 * PIECE, 14 * PIECE + 77, 8 * PIECE])
def test_v_between_its_tensors_and_in_their_memory(qgx, n, cut, make, kind):
    K, d = 3, (n + 3) // 4 * 4
    x = make(K, n, cut)
    ctx = qgx.Context(d, K, 256)
    limit = 1.5 * 2.0 ** 24 if make is half_way else 3.0
    offsets = [0, cut]

    apart = [torch.from_numpy(t.copy()).cuda() for t in (x[:, :cut], x[:, cut:])]
    fill = torch.full((K, d), 7.0, device="cuda")
    norms, V = clipped(qgx, ctx, apart, offsets, fill.clone(), limit, kind)

    # one tensor below V, the other above it
    room = torch.zeros(3 * K * d, device="cuda")
    low, mid, high = room[:K * cut].view(K, cut), room[K * d:2 * K * d].view(K, d), room[2 * K * d:2 * K * d + K * (n - cut)].view(K, n - cut)
    low.copy_(apart[0])
    high.copy_(apart[1])
    mid.copy_(fill)
    n2, V2 = clipped(qgx, ctx, [low, high], offsets, mid, limit, kind)
    assert np.array_equal(norms, n2) and np.array_equal(V, V2)

    # V between the first worker's elements of a tensor and the second's
    far = torch.zeros(K * (d * (K + 2)), device="cuda")
    step = d * (K + 1)
    spread = far.as_strided((K, cut), (step, 1), 0).copy_(apart[0])
    n3, V3 = clipped(qgx, ctx, [spread, apart[1]], offsets, far[d:d + K * d].view(K, d).copy_(fill), limit, kind)
    assert np.array_equal(norms, n3) and np.array_equal(V, V3)
    if make is half_way and kind == "l2":
        assert norms[0] == 2.0 ** 24 and norms[1] == 2.0 ** 25

    # V where one of its tensors lies, or both
    own = fill.clone()
    own[:, :cut], own[:, cut:n] = apart[0], apart[1]
    for tensors in ([own[:, :cut], own[:, cut:n]], [own[:, :cut], apart[1]], [apart[0], own[:, cut:n]]):
        twin = own.clone()
        n4, V4 = clipped(qgx, ctx, tensors, offsets, own, limit, kind)
        assert np.abs(n4 / norms.astype(np.float64) - 1).max() <= 2.0 ** -22 and (np.abs(V4 - V.astype(np.float64)) <= 2.0 ** -21 * np.abs(V)).all()
        own.copy_(twin)
    ctx.close()


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_tensors_of_16_bits_around_v(qgx, typ):
    K, n = 4, 5 * PIECE
    d = 2 * n
    ctx = qgx.Context(d, K, 256)
    x = torch.from_numpy(random(K, d)).cuda().to(TYPES[typ])
    norms, V = clipped(qgx, ctx, [x[:, :n].contiguous(), x[:, n:].contiguous()], [0, n], torch.zeros(K, d, device="cuda"), 5.0, "l2")
    room = torch.zeros(K * d * 2 + K * d, device="cuda")
    low, high = room[:K * n // 2].view(TYPES[typ]).view(K, n), room[2 * K * d:2 * K * d + K * n // 2].view(TYPES[typ]).view(K, n)
    low.copy_(x[:, :n])
    high.copy_(x[:, n:])
    n2, V2 = clipped(qgx, ctx, [low, high], [0, n], room[K * d:2 * K * d].view(K, d), 5.0, "l2")
    assert np.array_equal(norms, n2) and np.array_equal(V, V2)
    ctx.close()
