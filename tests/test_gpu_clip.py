"""Global gradient norm and clipping over many tensors (qgx_tensor_list_*, qgx_clip_gradients) against numpy in 64 bits.

Bounds: the norm is a sum of squares in binary64 (relative error below 2^-40 at these sizes), its root rounded to binary32:
2^-23 is more than that rounding.  An element is multiplied by a binary32 factor (2^-24, from a norm good to 2^-40) and rounded
(2^-24): 2^-22 together; in place a tensor of 16 bits is rounded to 11 or 8 bits of mantissa instead (2^-11, 2^-8)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {torch.float32: 2.0 ** -22, torch.float16: 2.0 ** -11 + 2.0 ** -22, torch.bfloat16: 2.0 ** -8 + 2.0 ** -22}
SIZES = [1, 3, 4, 7, 64, 0, 255, 8191, 8192, 8193, 20001, 5, 3 * 8192]


@pytest.fixture(scope="module")
def qgx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    m.load()
    return m


def up4(n):
    return (n + 3) // 4 * 4


def make(sizes, K, types, seed=1, scale=1.0, gap=3):
    """Tensors [K, n] inside wider, oddly placed memory; offsets with gaps of up to three coordinates."""
    g = np.random.default_rng(seed)
    tensors, offsets, at = [], [], 0
    for i, n in enumerate(sizes):
        x = (scale * g.standard_normal((K, n + gap)) * 10.0 ** g.uniform(-2, 1)).astype(np.float32)
        base = torch.from_numpy(x).cuda().to(types[i % len(types)])
        tensors.append(base[:, 1:1 + n])
        offsets.append(at)
        at += up4(n)
    return tensors, offsets, max(at, 4)


def want(tensors, offsets, d, limit, kind, fill):
    """Norms and V in 64 bits."""
    K = tensors[0].shape[0] if tensors else fill.shape[0]
    xs = [t.double().cpu().numpy() for t in tensors]
    with np.errstate(all="ignore"):
        if kind == "l2":
            norms = np.sqrt(sum((x * x).sum(1) for x in xs) if xs else np.zeros(K))
        else:
            norms = np.max(np.concatenate([np.zeros((K, 1))] + [np.abs(x) for x in xs], axis=1), axis=1)
        c = np.where(np.isfinite(norms) & (norms > limit), limit / norms, 1.0)
    V = fill.astype(np.float64).copy()
    for x, off in zip(xs, offsets):
        V[:, off:off + x.shape[1]] = x * c[:, None]
    return norms, c, V


def close(got, exact, rel):
    got, exact = np.asarray(got, np.float64), np.asarray(exact, np.float64)
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - exact) <= rel * np.abs(exact) + 1e-44) | (np.isnan(got) & np.isnan(exact)) | (got == exact))
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], exact[bad][:3])


@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["f32", "bf16", "f16"]])
@pytest.mark.parametrize("K,sizes", [(3, SIZES), (1, [1]), (2, [5]), (1, [70001]), (5, [17] * 150), (2, [1 << 20, 3, 300000])])
def test_gather_and_norm(qgx, K, sizes, types, kind):
    tensors, offsets, d = make(sizes, K, [TYPES[t] for t in types])
    fill = np.random.default_rng(7).standard_normal((K, d)).astype(np.float32)
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list(tensors, offsets)
    norms, _, _ = want(tensors, offsets, d, np.inf, kind, fill)
    for limit in (np.inf, float(np.float32(np.median(norms) * 0.7)), 0.0):
        V = torch.from_numpy(fill).cuda()
        got = ctx.clip_gradients(lst, limit, norm=qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF, out=V)
        norms, c, exact = want(tensors, offsets, d, limit, kind, fill)
        close(got.cpu().numpy(), norms, 2.0 ** -23)
        close(V.cpu().numpy(), exact, 2.0 ** -22)
        for k in np.flatnonzero(c == 1.0):                     # passed on unchanged, and coordinates of no tensor untouched
            assert np.array_equal(V[k].cpu().numpy(), exact[k].astype(np.float32))
    assert ctx.poll_error() == 0
    ctx.close()


@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["f16", "f32", "bf16"]])
def test_in_place(qgx, types):
    K = 3
    tensors, offsets, d = make(SIZES, K, [TYPES[t] for t in types])
    whole = [t._base.clone() if t._base is not None else t.clone() for t in tensors]
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list(tensors, offsets)
    xs = [t.double().cpu().numpy() for t in tensors]
    norms, _, _ = want(tensors, offsets, d, np.inf, "l2", np.zeros((K, d)))
    limit = float(np.float32(np.median(norms)))
    got = ctx.clip_gradients(lst, limit)
    close(got.cpu().numpy(), norms, 2.0 ** -23)
    c = np.where(norms > limit, limit / norms, 1.0)
    for t, x, w in zip(tensors, xs, whole):
        tiny = 2.0 ** -25 if t.dtype == torch.float16 else 0.0    # f16's subnormals: half their spacing
        y = t.double().cpu().numpy()
        assert (np.abs(y - x * c[:, None]) <= ROUND[t.dtype] * np.abs(x * c[:, None]) + tiny + 1e-44).all()
        if t._base is not None:                                   # nothing beside the tensors is written
            assert torch.equal(t._base[:, 0], w[:, 0]) and torch.equal(t._base[:, 1 + t.shape[1]:], w[:, 1 + t.shape[1]:])
    ctx.close()


def test_a_tensor_of_v_itself(qgx):
    K, d = 4, 4096 * 3 + 8
    V = torch.randn(K, d, device="cuda")
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list([V])
    norms, _, exact = want([V], [0], d, 50.0, "l2", np.zeros((K, d)))
    twin = V.clone()
    got = ctx.clip_gradients(lst, 50.0, out=V)
    close(got.cpu().numpy(), norms, 2.0 ** -23)
    close(V.cpu().numpy(), exact, 2.0 ** -22)
    lst2 = ctx.tensor_list([twin])
    ctx.clip_gradients(lst2, 50.0)
    assert torch.equal(V, twin)
    ctx.close()


def test_norm_at_the_limit_is_not_clipped(qgx):
    x = torch.zeros(2, 100, device="cuda")
    x[0, 3], x[0, 50] = 3.0, -4.0
    x[1, 9] = 5.0
    ctx = qgx.Context(100, 2, 256)
    lst = ctx.tensor_list([x])
    V = torch.empty(2, 100, device="cuda")
    n = ctx.clip_gradients(lst, 5.0, out=V)
    assert n.tolist() == [5.0, 5.0] and torch.equal(V, x)
    n = ctx.clip_gradients(lst, 2.5, out=V)
    assert torch.equal(V, 0.5 * x)
    ctx.close()


@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("poison", [np.nan, np.inf, -np.inf])
def test_non_finite_worker_passes_unscaled_and_is_reported(qgx, poison, kind):
    K = 3
    tensors, offsets, d = make([300, 9000, 5], K, [torch.float32, torch.bfloat16])
    tensors[1][1, 8999] = poison
    fill = np.zeros((K, d), np.float32)
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list(tensors, offsets)
    V = torch.zeros(K, d, device="cuda")
    norms, _, exact = want(tensors, offsets, d, 0.1, kind, fill)
    got = ctx.clip_gradients(lst, 0.1, norm=qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF, out=V)
    g = got.cpu().numpy()
    assert not np.isfinite(g[1]) and np.isfinite(g[[0, 2]]).all()
    close(g[[0, 2]], norms[[0, 2]], 2.0 ** -23)
    close(V.cpu().numpy(), exact, 2.0 ** -22)
    assert ctx.poll_error() == qgx.EBIT_NONFINITE and ctx.poll_error() == 0
    ctx.close()


def test_squares_beyond_binary32_and_below(qgx):
    x = torch.full((2, 1000), 1e30, device="cuda")
    x[1] = 1e-30
    ctx = qgx.Context(1000, 2, 256)
    lst = ctx.tensor_list([x])
    V = torch.empty(2, 1000, device="cuda")
    n = ctx.clip_gradients(lst, 1e-29, out=V).double().cpu().numpy()
    x64 = x.double().cpu().numpy()
    norms = np.sqrt((x64 * x64).sum(1))
    close(n, norms, 2.0 ** -23)
    close(V.double().cpu().numpy(), x64 * (np.float32(1e-29).astype(np.float64) / norms)[:, None], 2.0 ** -21)
    assert ctx.poll_error() == 0
    ctx.close()


def test_empty_lists_and_tensors(qgx):
    ctx = qgx.Context(64, 2, 256)
    V = torch.ones(2, 64, device="cuda")
    for tensors in ([], [torch.empty(2, 0, device="cuda")], [torch.empty(2, 0, device="cuda")] * 3):
        n = ctx.clip_gradients(ctx.tensor_list(tensors), 1.0, out=V)
        assert n.tolist() == [0.0, 0.0] and bool((V == 1).all())
        assert ctx.clip_gradients(ctx.tensor_list(tensors), 1.0).tolist() == [0.0, 0.0]
    ctx.close()


def test_workers_that_share_a_gradient(qgx):
    x = torch.randn(1, 500, device="cuda").expand(3, 500)
    ctx = qgx.Context(500, 3, 256)
    lst = ctx.tensor_list([x])
    V = torch.empty(3, 500, device="cuda")
    n = ctx.clip_gradients(lst, 1.0, out=V)
    close(n.cpu().numpy(), np.linalg.norm(x.double().cpu().numpy(), axis=1), 2.0 ** -23)
    assert torch.equal(V[0], V[1]) and torch.equal(V[0], V[2])
    with pytest.raises(qgx.QgxError) as e:
        ctx.clip_gradients(lst, 1.0)
    assert e.value.status == qgx.ERR_ARG
    ctx.close()


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", ["l2", "linf"])
@pytest.mark.parametrize("sizes", [[5 * 4096], [20000, 3], [30, 7, 4096, 1, 9, 4097, 2], [8 * 4096 + 1], [65536], [4096] * 16, [5] * 17])
def test_some_pieces(qgx, sizes, kind, typ):
    K = 3
    tensors, offsets, d = make(sizes, K, [TYPES[typ]])
    c = qgx.Context(d, K, 256)
    lst, fill = c.tensor_list(tensors, offsets), np.full((K, d), 7.0)
    norms, _, _ = want(tensors, offsets, d, np.inf, kind, fill)
    limit = float(np.float32(np.median(norms) * 0.9))
    norms, _, exact = want(tensors, offsets, d, limit, kind, fill)
    V = torch.full((K, d), 7.0, device="cuda")
    close(c.clip_gradients(lst, limit, norm=qgx.NORM_L2 if kind == "l2" else qgx.NORM_LINF, out=V).cpu().numpy(), norms, 2.0 ** -23)
    close(V.cpu().numpy(), exact, 2.0 ** -22)
    c.close()


@pytest.mark.parametrize("shift", [0, 40960])
def test_v_in_the_memory_of_its_tensors(qgx, shift):
    """A tensor that lies where V has it, of as many pieces as a workgroup reads for itself elsewhere."""
    K, n = 2, 40960
    d = n + shift
    c = qgx.Context(d, K, 256)
    V = torch.from_numpy(np.random.default_rng(1).standard_normal((K, d)).astype(np.float32)).cuda()
    tensors, offsets = [V[:, shift:]], [shift]
    norms, _, exact = want(tensors, offsets, d, 2.0, "l2", V.double().cpu().numpy())
    lst = c.tensor_list(tensors, offsets)
    close(c.clip_gradients(lst, 2.0, out=V).cpu().numpy(), norms, 2.0 ** -23)
    close(V.cpu().numpy(), exact, 2.0 ** -22)
    c.close()


def test_offsets_beyond_32_bits(qgx):
    K, n, far = 2, 50001, (1 << 32) + 24                     # workers' tensors four thousand million elements apart
    memory = torch.empty(far + (1 << 20), device="cuda", dtype=torch.bfloat16)
    tensors = [memory.as_strided((K, n), (far, 1), at) for at in (1, 300001)]
    for i, t in enumerate(tensors):
        t.copy_(torch.from_numpy(np.random.default_rng(i).standard_normal((K, n))))
    offsets, d = [0, up4(n)], 2 * up4(n)
    c = qgx.Context(d, K, 256)
    norms, scale, V = want(tensors, offsets, d, 3.0, "l2", np.full((K, d), 7.0))
    lst, got = c.tensor_list(tensors, offsets), torch.full((K, d), 7.0, device="cuda")
    close(c.clip_gradients(lst, 3.0, out=got).cpu(), norms, 2 * 2.0 ** -24)
    close(got.cpu(), V, 2 * 2.0 ** -24)
    before = [t.clone() for t in tensors]
    c.clip_gradients(lst, 3.0)
    for t, x in zip(tensors, before):
        close(t.double().cpu().numpy(), x.double().cpu().numpy() * scale[:, None], (2.0 ** -8 + 2.0 ** -24) * 1.001)
    c.close()


def test_repeats_bit_for_bit_and_on_another_stream(qgx):
    K = 4
    tensors, offsets, d = make([300001, 40, 70000], K, [torch.float32, torch.bfloat16])
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list(tensors, offsets)
    a, b = torch.zeros(K, d, device="cuda"), torch.zeros(K, d, device="cuda")
    na = ctx.clip_gradients(lst, 1.0, out=a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    nb = ctx.clip_gradients(lst, 1.0, out=b, stream=s)
    s.synchronize()
    assert torch.equal(a, b) and torch.equal(na, nb)
    ctx.close()


def test_captured_graph_replays(qgx):
    K, d = 2, 50000
    x = torch.randn(K, d, device="cuda")
    V = torch.zeros(K, d, device="cuda")
    ctx = qgx.Context(d, K, 256)
    lst = ctx.tensor_list([x])
    ctx.clip_gradients(lst, 3.0, out=V)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        n = ctx.clip_gradients(lst, 3.0, out=V)
    for i in range(4):
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        twin = torch.zeros_like(V)
        eager = ctx.clip_gradients(lst, 3.0, out=twin)
        assert torch.equal(V, twin) and torch.equal(n, eager)
    ctx.close()


def test_refusals(qgx):
    ctx = qgx.Context(100, 2, 256)
    x = torch.zeros(2, 60, device="cuda")
    V = torch.zeros(2, 100, device="cuda")

    def refused(f, status=qgx.ERR_ARG):
        with pytest.raises(qgx.QgxError) as e:
            f()
        assert e.value.status == status and str(e.value)

    refused(lambda: ctx.tensor_list([x, x]))                              # 120 coordinates of 100
    refused(lambda: ctx.tensor_list([x, x], [0, 30]))                     # overlap in V
    refused(lambda: ctx.tensor_list([x], [41]))
    refused(lambda: ctx.tensor_list([x], [0, 1]))
    refused(lambda: ctx.tensor_list([x.double()]))
    refused(lambda: ctx.tensor_list([x.cpu()]))
    refused(lambda: ctx.tensor_list([x[:1]]))                             # one worker's rows for two
    refused(lambda: ctx.tensor_list([torch.zeros(2, 120, device="cuda")[:, ::2]]))
    lst = ctx.tensor_list([x])
    refused(lambda: ctx.clip_gradients(lst, -1.0, out=V))
    refused(lambda: ctx.clip_gradients(lst, float("nan"), out=V))
    refused(lambda: ctx.clip_gradients(lst, 1.0, norm=1, out=V))
    refused(lambda: ctx.clip_gradients(lst, 1.0, out=V[:, :99]))
    refused(lambda: ctx.clip_gradients(lst, 1.0, out=V.double()))
    other = qgx.Context(60, 2, 256)
    refused(lambda: other.clip_gradients(lst, 1.0))                       # made for 100 coordinates
    other.close()
    lst._c.table_bytes -= 8
    refused(lambda: ctx.clip_gradients(lst, 1.0, out=V), qgx.ERR_CAPACITY)
    ctx.close()
