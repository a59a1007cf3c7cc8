"""Group norm backward (qgx_group_norm_backward): groups whose neighbours are no numbers or far larger."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": U, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256, seed=78)
    yield c
    c.close()


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("batch", [1, 70])
def test_small_groups_beside_far_larger_ones(ctx, typ, batch):
    """Groups that share a block of 32, one of values so large that the block's step times another's rstd is beyond binary32: the small ones were kept as zeros,
    h = -mean rstd.  One place, groups of one piece.  h is off by 3 u of itself, sums of n terms by n u of their magnitudes, dx by four roundings more."""
    n = 4 if typ == "f32" else 8
    C, G = 32, 32 // n
    g = torch.Generator(device="cuda")
    g.manual_seed(batch)
    x = torch.randn(1, batch, 1, C, generator=g, device="cuda") * 1e-3
    x[..., :n] = 3.3e38 / n
    x = x.to(TYPES[typ])
    dy = torch.randn(x.shape, generator=g, device="cuda").to(TYPES[typ])
    y, mean, rstd = ctx.group_norm(x, G)
    assert bool(torch.isfinite(y).all()) and bool(torch.isfinite(rstd).all())
    kept = ctx.checkpoint(x)
    assert float(ctx.restore(kept)[..., n:].abs().max()) == 0
    dw, db = torch.empty(1, C, device="cuda"), torch.empty(1, C, device="cuda")
    dx = ctx.group_norm_backward(dy, kept, G, None, None, mean, rstd, dw=dw, db=db)
    v, d = (t.double().cpu().numpy().reshape(batch, G, n)[:, 1:] for t in (ctx.restore(kept), dy))
    mu, r = (t.double().cpu().numpy().reshape(batch, G, 1)[:, 1:] for t in (mean, rstd))
    h = (v - mu) * r
    m1, m2 = d.mean(-1, keepdims=True), (d * h).mean(-1, keepdims=True)
    a1, a2 = np.abs(d).mean(-1, keepdims=True), np.abs(d * h).mean(-1, keepdims=True)
    want = (d - m1 - h * m2) * r
    err = (16 + n) * U * r * (np.abs(d) + a1 + np.abs(h) * a2)
    err = err + ROUND[typ] * (np.abs(want) + err)
    assert (np.abs(dx.double().cpu().numpy().reshape(batch, G, n)[:, 1:] - want) <= err).all()
    terms = np.abs(d * h).sum(0).reshape(-1)
    assert (np.abs(dw.double().cpu().numpy()[0, n:] - (d * h).sum(0).reshape(-1)) <= (batch + 8) * U * terms).all()
    for kind in ("silu", "leaky"):
        assert bool(torch.isfinite(ctx.group_norm_backward(dy, kept, G, None, None, mean, rstd, kind)[..., n:]).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, 3 * 2.0 ** 121])
@pytest.mark.parametrize("kind", ["none", "silu", "leaky"])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("batch,P,C,G", [(2, 50, 64, 8), (2, 30, 128, 8), (600, 3, 64, 8), (1100, 3, 64, 8), (2, 9000, 64, 8)])
def test_a_groups_gradient_is_its_own(ctx, batch, P, C, G, typ, kind, bad):
    """From kept codes and from x: what a group of another block of 32 holds, no numbers or one far value throughout, leaves every bit of the others."""
    g = torch.Generator(device="cuda")
    g.manual_seed(P)
    x, dy = (torch.randn(1, batch, P, C, generator=g, device="cuda").to(TYPES[typ]) for _ in range(2))
    w, b = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    _, mean, rstd = ctx.group_norm(x, G, w, b, activation=kind)
    spoilt, m, r = x.clone(), mean.clone(), rstd.clone()
    spoilt[..., C - C // G:] = bad                         # the last group, in the last block
    m[..., -1] = bad
    r[..., -1] = 1e5 ** 0.5 if math.isfinite(bad) else math.nan
    for keep in (False, True):
        got = []
        for source, mu, rs in ((x, mean, rstd), (spoilt, m, r)):
            dw, db = torch.empty(1, C, device="cuda"), torch.empty(1, C, device="cuda")
            dx = ctx.group_norm_backward(dy, ctx.checkpoint(source, 2) if keep else source, G, w, b, mu, rs, kind, dw=dw, db=db)
            got.append([t[..., :C - 32] for t in (dx, dw, db)])
        assert all(torch.equal(s, t) for s, t in zip(*got))
        assert bool(torch.isfinite(got[1][0]).all())
    ctx.poll_error()
