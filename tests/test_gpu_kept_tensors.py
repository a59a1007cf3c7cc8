"""Several activations kept in one call of the method: each has a number of its own in the draws, so that what they are rounded by is independent.

An element's draw is 16 bits of Philox4x32-10 at (column / 8, 2 + 256 tensor, row, call); the codes are compared for equality with a model in whole numbers."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SEED = 0x0123456789ABCDEF
MOST = (1 << 24) - 1


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 3, 256, seed=SEED)
    yield c
    c.close()


def draws(rows, cols, call, tensor):
    groups = (cols + 7) // 8
    m32 = np.uint64(0xFFFFFFFF)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.full(rows * groups, 2 + 256 * tensor, np.uint64), np.repeat(np.arange(rows, dtype=np.uint64), groups),
         np.full(rows * groups, call, np.uint64)]
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack([x.astype(np.uint32) for x in c], 1)
    return np.stack([w & 0xFFFF, w >> 16], 2).reshape(rows, groups * 8)[:, :cols]


def check(x, kept, call, tensor):
    """The codes of x [.., cols], with the blocks' powers as they were kept (numbers of ordinary size)."""
    cols = x.shape[-1]
    v = x.double().cpu().numpy().reshape(-1, cols)
    powers = kept.powers.cpu().numpy().reshape(v.shape[0], -1).astype(int)
    u = np.ldexp(v, 127 - powers.repeat(32, 1)[:, :cols])
    m = np.abs(u)
    want = np.sign(u) * (np.floor(m) + (draws(v.shape[0], cols, call, tensor) < (m - np.floor(m)) * 65536.0))
    assert np.array_equal(kept.codes.cpu().numpy().reshape(v.shape[0], -1)[:, :cols].astype(int) - 128, want.astype(int))


@pytest.mark.parametrize("tensor", [0, 1, 2, 77, MOST])
@pytest.mark.parametrize("typ", TYPES)
def test_a_tensors_number_is_in_its_draws(ctx, typ, tensor):
    for shape in ((5, 100), (3, 7, 64), (2, 3, 40, 33)):
        x = torch.randn(shape, device="cuda").to(TYPES[typ])
        kept = ctx.checkpoint(x, 9, tensor=tensor)
        assert kept.tensor == tensor
        check(x, kept, 9, tensor)
        out = ctx.new_checkpoint(shape, tensor=tensor)
        assert ctx.checkpoint(x, 9, out=out) is out and torch.equal(out.codes, kept.codes)


@pytest.mark.parametrize("tensor", [0, 3, MOST])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("P,C,G", [(64, 64, 8), (9, 45, 5), (9000, 32, 4)])
def test_group_norm_keeps_by_it_too(ctx, P, C, G, typ, tensor):
    x = torch.randn(2, 2, P, C, device="cuda").to(TYPES[typ])
    kept = ctx.new_checkpoint(x.shape, tensor=tensor)
    ctx.group_norm(x, G, keep=kept, call_id=4)
    alone = ctx.checkpoint(x, 4, tensor=tensor)
    assert torch.equal(kept.codes, alone.codes) and torch.equal(kept.powers, alone.powers)
    if P <= 64:
        check(x, kept, 4, tensor)


def test_to_nearest_it_does_not_matter(ctx):
    x = torch.randn(9, 77, device="cuda")
    assert torch.equal(ctx.checkpoint(x, tensor=5).codes, ctx.checkpoint(x).codes)


def test_tensors_of_one_half_step_in_a_graph(ctx):
    """The iteration's own call numbers: two tensors of a half-step still differ, at every replay."""
    from paper_2308_09187_amd import qgx, synth
    c = qgx.Context(4096, 2, 256, seed=SEED)
    c.set_levels(synth.levels_exponential(8))
    c.state_init()
    V = torch.randn(2, 4096, device="cuda")
    s = c.new_stream()
    c.quantize_encode(V, 0, s)
    x = torch.randn(6, 100, device="cuda")
    kept = [c.new_checkpoint(x.shape, tensor=t) for t in (1, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        for k in kept:
            c.checkpoint(x, qgx.CALL_SECOND_HALF, out=k, stream=side)
    for t in range(3):
        g.replay()
        torch.cuda.synchronize()
        for k in kept:
            check(x, k, 2 * t + 1, k.tensor)
        assert not torch.equal(kept[0].codes, kept[1].codes)
        c.eg_step(1, s, None)
        x.add_(1.0)
    c.close()


def test_a_product_of_two_kept_tensors_has_its_expectation(ctx):
    """The mean over n calls of the product of both errors, each within a step s of its block, is by Hoeffding off 0 by more than 2 s^2 sqrt(ln(2 / 1e-12) / 2 n)
    with probability 1e-12 an element, 64 of them; the draws' 16 bits add 2 s^2 2^-16.  (By the same draws it would be up to s^2 / 4.)"""
    x = torch.linspace(-1.0, 1.0, 64, device="cuda").view(1, 64) * 0.77
    n = 2000
    total = torch.zeros(1, 64, device="cuda", dtype=torch.float64)
    for call in range(n):
        a, b = (ctx.restore(ctx.checkpoint(x, call, tensor=t)).double() - x.double() for t in (0, 1))
        total += a * b
    step = torch.exp2(ctx.checkpoint(x).powers.view(2).double() - 127.0).repeat_interleave(32)
    bound = 2 * step ** 2 * (math.sqrt(math.log(2e12) / (2 * n)) + 2.0 ** -16)
    assert bool(((total / n).abs() <= bound).all())


def test_refusals(ctx):
    from paper_2308_09187_amd import qgx
    x = torch.zeros(4, 40, device="cuda")
    k = ctx.checkpoint(x)

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    for bad in (-1, MOST + 1):
        refused(lambda: ctx.checkpoint(x, 1, tensor=bad))
        refused(lambda: ctx.new_checkpoint(x.shape, tensor=bad))
        refused(lambda: qgx.Checkpoint(k.codes, k.powers, 40, tensor=bad))
    refused(lambda: ctx.checkpoint(x, 1, out=k, tensor=1))            # out has a number of its own
    assert qgx.Checkpoint(k.codes, k.powers, 40, tensor=MOST).tensor == MOST and k.tensor == 0
    k._c.tensor = MOST + 1
    refused(lambda: ctx.checkpoint(x, 1, out=k))
    refused(lambda: ctx.group_norm(x, 4, keep=k, call_id=1))
    assert torch.equal(ctx.restore(k), x)                  # (what was kept is read without it)
