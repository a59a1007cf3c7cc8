"""Clipping at sizes where a workgroup sums several pieces and where the scaling launch takes the factors that another one left, into V and in
place, in both norms; and the largest magnitude in place in every form.

Bounds: an element is multiplied in binary64 by a factor good to 2^-50 (squares in binary64 in a tree of at most 2^11 terms a thread) and rounded to binary32:
2^-24 and a little (or half the spacing 2^-149 of its subnormal numbers); in place that is rounded to 11 or 8 bits as well: 2^-11, 2^-8, or half
the spacing of the subnormal numbers there, 2^-25 and 2^-134."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_clip import make, qgx, want  # noqa: E402, F401

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SINGLE = 2.0 ** -24 * (1 + 2.0 ** -20)
IN_PLACE = {torch.float32: (SINGLE, 2.0 ** -150), torch.float16: (2.0 ** -11 + SINGLE, 2.0 ** -25), torch.bfloat16: (2.0 ** -8 + SINGLE, 2.0 ** -134)}
PIECE = 4096
MANY = [PIECE * 150 + 17, 3, PIECE * 99 + 4095, 1, 0, 7, 20001, PIECE, 5]


def within(got, exact, rel, least):
    err = np.abs(got.astype(np.float64) - exact)
    assert (err <= rel * np.abs(exact) + least).all(), np.argwhere(err > rel * np.abs(exact) + least)[:3]


def setup(qgx, sizes, K, types, kind):  # noqa: F811
    """Tensors, one worker's far smaller than the others', and a limit between."""
    tensors, offsets, d = make(sizes, K, types)
    if K > 1:
        for t in tensors:
            t[K - 1] *= 2.0 ** -6
    fill = np.full((K, d), 7.0, np.float32)
    norms, _, _ = want(tensors, offsets, d, np.inf, kind, fill)
    limit = float(np.float32(np.median(norms[:max(1, K - 1)]) * 0.8))
    norms, c, V = want(tensors, offsets, d, limit, kind, fill)
    assert (c < 1).any() and (K == 1 or c[K - 1] == 1.0)
    return tensors, offsets, d, limit, norms, c, V


@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["f32", "bf16", "f16"]])
@pytest.mark.parametrize("K,sizes", [(8, MANY), (2, MANY * 5), (3, [PIECE * 1100 + 1]), (40, [70001, 5])])
def test_many_pieces(qgx, K, sizes, types, kind):  # noqa: F811
    tensors, offsets, d, limit, norms, c, exact = setup(qgx, sizes, K, [TYPES[t] for t in types], kind)
    before = [t.double().cpu().numpy() for t in tensors]
    margins = [(t._base[:, 0].clone(), t._base[:, 1 + t.shape[1]:].clone()) for t in tensors]
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list(tensors, offsets)
    which = qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF
    V = torch.full((K, d), 7.0, device="cuda")
    within(ctx.clip_gradients(lst, limit, norm=which, out=V).cpu().numpy(), norms, SINGLE, 0.0)
    got = V.cpu().numpy()
    within(got, exact, SINGLE, 2.0 ** -150)
    for k in np.flatnonzero(c == 1.0):                         # passed on unchanged
        assert np.array_equal(got[k], exact[k].astype(np.float32))
    within(ctx.clip_gradients(lst, limit, norm=which).cpu().numpy(), norms, SINGLE, 0.0)
    for t, x, (left, right) in zip(tensors, before, margins):
        y = t.double().cpu().numpy()
        within(y, x * c[:, None], *IN_PLACE[t.dtype])
        for k in np.flatnonzero(c == 1.0):
            assert np.array_equal(y[k], x[k])
        assert torch.equal(t._base[:, 0], left) and torch.equal(t._base[:, 1 + t.shape[1]:], right)
    assert ctx.poll_error() == 0
    ctx.close()


@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["f16", "f32", "bf16"]])
@pytest.mark.parametrize("sizes", [[5], [3 * PIECE + 1], [100, 4097, 3], [10 * PIECE + 9, 2], [20 * PIECE, 40001, 77]])
def test_few_pieces_in_place(qgx, sizes, types, kind):  # noqa: F811
    K = 3
    tensors, offsets, d, limit, norms, c, _ = setup(qgx, sizes, K, [TYPES[t] for t in types], kind)
    before = [t.double().cpu().numpy() for t in tensors]
    ctx = qgx.Context(d, K, 256)
    within(ctx.clip_gradients(ctx.tensor_list(tensors, offsets), limit, norm=qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF).cpu().numpy(), norms, SINGLE, 0.0)
    for t, x in zip(tensors, before):
        y = t.double().cpu().numpy()
        within(y, x * c[:, None], *IN_PLACE[t.dtype])
        for k in np.flatnonzero(c == 1.0):
            assert np.array_equal(y[k], x[k])
    ctx.close()
