"""Activations kept in 8 bits (qgx_checkpoint, qgx_restore) against their definition, code by code.

Every step is exact (a power of two divides out, a remainder of at most 24 bits is compared with 16), so all is compared for equality; the model below works
in numpy's binary64 and whole numbers, with a Philox of its own."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SEED = 0x9876543210FEDCBA
COLS = [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 255, 256, 1000, 1001, 4096, 8197]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 3, 256, seed=SEED)
    yield c
    c.close()


def draws(rows, cols, call, seed=SEED):
    groups = (cols + 7) // 8
    m32 = np.uint64(0xFFFFFFFF)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.full(rows * groups, 2, np.uint64), np.repeat(np.arange(rows, dtype=np.uint64), groups),
         np.full(rows * groups, call, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack([x.astype(np.uint32) for x in c], 1)
    return np.stack([w & 0xFFFF, w >> 16], 2).reshape(rows, groups * 8)[:, :cols]


def model(x, typ, call):
    """codes, powers, values of x [rows, cols] in binary64."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    v = np.zeros((rows, blocks * 32))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, 32)
    finite = np.isfinite(v).all(2)
    v = np.where(finite[..., None], v, 0.0)
    top = np.abs(v).max(2)
    e = np.zeros((rows, blocks), int)
    for i in np.ndindex(rows, blocks):
        if top[i]:
            f, n = math.frexp(top[i])                      # top = f 2^n, 1/2 <= f < 1; 127 = 0.9921875 * 2^7
            e[i] = n - 7 + (f > 0.9921875)
    e = np.clip(e, -126, 9 if typ == "f16" else 121)
    u = np.ldexp(v, -e[..., None])
    if call is None:
        c = np.rint(u)
    else:
        r = np.zeros((rows, blocks * 32))
        r[:, :cols] = draws(rows, cols, call)
        m = np.abs(u)
        c = np.sign(u) * (np.floor(m) + (r.reshape(v.shape) < (m - np.floor(m)) * 65536.0))
    c = np.clip(c, -127, 127)
    powers = np.where(finite, np.where(top == 0, 0, e + 127), 255)
    c = np.where(powers[..., None] == 0, 0, c)
    values = np.where(finite[..., None], np.ldexp(c, e[..., None]), np.nan)
    return (c + 128).astype(np.uint8).reshape(rows, -1), powers.astype(np.uint8), values.reshape(rows, -1)[:, :cols]


def inputs(seed, rows, cols, typ):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-12, 8, (rows, 1)))
    x[g.random((rows, cols)) < 0.1] = 0.0
    return torch.from_numpy(x).cuda().to(TYPES[typ])


def check(ctx, x, typ, call, kept=None):
    """x [.., cols] on the GPU."""
    kept = ctx.checkpoint(x, call) if kept is None else kept
    flat = x.double().cpu().numpy().reshape(-1, x.shape[-1])
    codes, powers, values = model(flat, typ, call)
    assert np.array_equal(kept.powers.cpu().numpy().reshape(powers.shape), powers)
    assert np.array_equal(kept.codes.cpu().numpy().reshape(codes.shape), codes)
    for t in TYPES.values():
        got = ctx.restore(kept, t)
        want = torch.from_numpy(values).to(torch.float32).to(t)          # (binary32 holds every value)
        assert got.shape == x.shape and torch.equal(got.cpu().view(values.shape).nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("call", [None, 5])
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows(ctx, cols, typ, call):
    check(ctx, inputs(cols, 5, cols, typ), typ, call)


@pytest.mark.parametrize("shape", [(1, 64), (700, 33), (3, 1, 129), (3, 41, 200), (2, 3, 5, 40), (2, 7, 1, 8), (1000, 8)])
def test_leading_dimensions(ctx, shape):
    x = inputs(1, math.prod(shape[:-1]), shape[-1], "bf16").view(shape)
    check(ctx, x, "bf16", 3)


@pytest.mark.parametrize("typ", TYPES)
def test_strides_and_odd_addresses(ctx, typ):
    big = inputs(2, 3 * 11, 201, typ).view(3, 11, 201)
    check(ctx, big[:, 1:8, 1:100], typ, 9)
    check(ctx, big.transpose(0, 1)[..., 7:], typ, None)
    check(ctx, big[:1].expand(3, 11, 201), typ, 9)          # (read only: rows may coincide)
    out = torch.full((33, 230), 5.0, device="cuda", dtype=TYPES[typ])
    kept = ctx.checkpoint(big.view(33, 201))
    ctx.restore(kept, out=out[:, 3:204])
    assert torch.equal(out[:, 3:204], ctx.restore(kept, TYPES[typ])) and bool((out[:, :3] == 5).all()) and bool((out[:, 204:] == 5).all())


@pytest.mark.parametrize("call", [None, 1])
@pytest.mark.parametrize("typ", TYPES)
def test_edges_of_the_range(ctx, typ, call):
    info = torch.finfo(TYPES[typ])
    x = torch.zeros(12, 64, dtype=torch.float64)
    x[0, :5] = torch.tensor([info.max, -info.max, info.max / 3, 1.0, 0.0])
    x[1, :4] = torch.tensor([info.tiny, -info.tiny, info.tiny / 2, 0.0])
    x[2, 0] = info.smallest_normal * 2.0 ** (-10 if typ == "f16" else -7 if typ == "bf16" else -23)          # the smallest number
    x[3, :3] = torch.tensor([127.0, 126.5, 0.5])           # ties, and the largest magnitude at a power's border
    x[4, :3] = torch.tensor([127.5, 1.0, -1.0])
    x[5, :2] = torch.tensor([-0.0, 0.0])
    x[6, :32] = torch.arange(32) - 16.5
    x[7, 40] = 1.0                                         # one block of zeros, one not
    x = x.cuda().to(TYPES[typ])
    check(ctx, x, typ, call)
    back = ctx.restore(ctx.checkpoint(x, call), TYPES[typ])
    assert bool(torch.isfinite(back).all()) and ctx.poll_error() == 0


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("typ", TYPES)
def test_no_numbers_spoil_their_block_and_are_reported(ctx, typ, bad):
    from paper_2308_09187_amd import qgx
    x = inputs(3, 4, 100, typ)
    x[2, 37] = bad
    ctx.poll_error()
    for call in (None, 2):
        check(ctx, x, typ, call)
        assert ctx.poll_error() == qgx.EBIT_NONFINITE
    got = torch.isnan(ctx.restore(ctx.checkpoint(x)))
    assert got[2, 32:64].all() and int(got.sum()) == 32
    ctx.poll_error()


def test_without_bias(ctx):
    """The mean over calls of what is kept: by Hoeffding off by more than sqrt(ln(2 / 1e-12) / 2 n) steps with probability 1e-12 an
    element, 64 of them; the draws' 16 bits add 2^-16."""
    x = torch.linspace(-1.0, 1.0, 64, device="cuda").view(1, 64).repeat(1, 1) * 0.77
    n = 4000
    total = torch.zeros(1, 64, device="cuda", dtype=torch.float64)
    for call in range(n):
        total += ctx.restore(ctx.checkpoint(x, call)).double()
    step = torch.ldexp(torch.ones(2, device="cuda", dtype=torch.float64), ctx.checkpoint(x).powers.view(2).int() - 127).repeat_interleave(32)
    bound = math.sqrt(math.log(2e12) / (2 * n)) + 2.0 ** -16
    assert bool((((total / n - x).abs() / step) <= bound).all())


def test_the_iterations_own_call_numbers_in_a_graph(ctx):
    """CALL_FIRST_HALF and CALL_SECOND_HALF: 2(t-1) and 2(t-1)+1 from the counter on the device, fresh at every replay."""
    from paper_2308_09187_amd import qgx, synth
    c = qgx.Context(4096, 2, 256, seed=SEED)
    c.set_levels(synth.levels_exponential(8))
    c.state_init()
    V = torch.randn(2, 4096, device="cuda")
    s = c.new_stream()
    c.quantize_encode(V, 0, s)
    x = inputs(4, 6, 100, "bf16")
    first, second = c.new_checkpoint(x.shape), c.new_checkpoint(x.shape)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.checkpoint(x, qgx.CALL_FIRST_HALF, out=first, stream=side)
        c.checkpoint(x, qgx.CALL_SECOND_HALF, out=second, stream=side)
    for t in range(4):
        g.replay()
        torch.cuda.synchronize()
        assert c.scalars()["t"] == t + 1
        check(c, x, "bf16", 2 * t, first)
        check(c, x, "bf16", 2 * t + 1, second)
        c.eg_step(1, s, None)
        x.add_(1.0)
    c.close()


def test_another_stream_repeats_and_nothing_to_do(ctx):
    x = inputs(5, 300, 777, "f32")
    want = ctx.checkpoint(x, 11)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ctx.checkpoint(x, 11, stream=side)
    back = ctx.restore(got, stream=side)
    side.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got.powers, want.powers) and torch.equal(back, ctx.restore(want))
    empty = ctx.checkpoint(torch.zeros(0, 40, device="cuda"))
    assert empty.codes.shape == (0, 64) and ctx.restore(empty).shape == (0, 40)
    assert ctx.restore(ctx.checkpoint(torch.zeros(2, 0, 40, device="cuda"))).shape == (2, 0, 40)


@pytest.mark.parametrize("call", [None, 3])
def test_offsets_beyond_32_bits(ctx, call):
    rows, cols, last = (1 << 20) + 9, 4128, 70
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-last:] = inputs(11, last, cols, "bf16")
    kept = ctx.checkpoint(x, call)
    flat = x[-last:].double().cpu().numpy()
    if call is None:
        codes, powers, values = model(flat, "bf16", None)
        assert np.array_equal(kept.codes[-last:].cpu().numpy(), codes) and np.array_equal(kept.powers[-last:].cpu().numpy(), powers)
        got = ctx.restore(kept, torch.float32)[-last:]
        assert np.array_equal(got.double().cpu().numpy(), values)
    else:                                                  # (to the one or the other side; the row in the draws is that of the whole)
        got = ctx.restore(kept, torch.float32)[-last:].double().cpu().numpy()
        step = np.exp2(kept.powers[-last:].double().cpu().numpy() - 127.0).repeat(32, 1)
        assert (np.abs(got - flat) < np.where(flat == 0, 1e-300, step)).all()
    assert int(kept.powers[:-last].max()) == 0 and int((kept.codes[:-last] != 128).sum()) == 0
    del x, kept, got
    torch.cuda.empty_cache()


def test_refusals(ctx):
    from paper_2308_09187_amd import qgx
    x = torch.zeros(4, 40, device="cuda")
    k = ctx.checkpoint(x)

    def refused(f):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == qgx.ERR_ARG and str(e.value)

    refused(lambda: ctx.checkpoint(x.double()))
    refused(lambda: ctx.checkpoint(x.cpu()))
    refused(lambda: ctx.checkpoint(x[:, ::2]))
    refused(lambda: ctx.checkpoint(x, call_id=-1))
    refused(lambda: ctx.checkpoint(x, call_id=1 << 32))
    refused(lambda: ctx.checkpoint(x, out=ctx.new_checkpoint((4, 41))))
    refused(lambda: ctx.checkpoint(x, out=ctx.new_checkpoint((5, 40))))
    refused(lambda: ctx.checkpoint(torch.zeros(2, 3, 4, 5, 8, device="cuda").permute(3, 0, 2, 1, 4)))
    refused(lambda: ctx.new_checkpoint((4, 0)))
    refused(lambda: ctx.restore(k, torch.float64))
    refused(lambda: ctx.restore(k, out=torch.zeros(4, 40, device="cuda", dtype=torch.float64)))
    refused(lambda: ctx.restore(k, out=torch.zeros(4, 41, device="cuda")))
    refused(lambda: ctx.restore(k, out=torch.zeros(1, 40, device="cuda").expand(4, 40)))
    refused(lambda: ctx.restore(k, out=torch.zeros(4, 80, device="cuda")[:, ::2]))
    refused(lambda: qgx.Checkpoint(k.codes.cpu(), k.powers.cpu(), 40))
    refused(lambda: qgx.Checkpoint(k.codes, k.powers, 33 + 64))
    refused(lambda: qgx.Checkpoint(k.codes[:, :40], k.powers, 40))
    refused(lambda: qgx.Checkpoint(k.codes.view(torch.int8), k.powers, 40))
    refused(lambda: qgx.Checkpoint(k.codes[:2], k.powers, 40))
    off = torch.zeros(4 * 64 + 1, device="cuda", dtype=torch.uint8)[1:].view(4, 64)
    refused(lambda: ctx.checkpoint(x, out=qgx.Checkpoint(off, k.powers, 40)))         # codes not aligned
