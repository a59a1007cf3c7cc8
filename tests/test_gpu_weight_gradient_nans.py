"""The weight gradient (qgx_weight_gradient) of a dy with NaNs of every payload: they spoil their column and no other."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BITS = {"f32": torch.int32, "f16": torch.int16, "bf16": torch.int16}
# NaNs, quiet and signalling, of high and of low payloads (a binary32's low 16 bits lie behind those of a bfloat16)
NANS = {"f32": [0x7F800001, -0x7FFFFF, 0x7F80FFFF, 0x7FA00000, 0x7FC00000], "f16": [0x7C01, -0x3FF, 0x7E00], "bf16": [0x7F81, -0x7F, 0x7FC0]}


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


@pytest.mark.parametrize("out", [1, 3, 140])
@pytest.mark.parametrize("typ", TYPES)
def test_nans_of_every_payload(ctx, typ, out):
    """Alone in a column, beside an infinity among the same eight rows (of one sign with the products, so that infinities alone would give one), and in rows past
    the last full step."""
    rows, cols = 197, 70
    x, dy = whole_numbers(3, 1, rows, cols, out, typ)
    x = x.abs() + 1.0
    kept, clean = ctx.checkpoint(x), product(x, dy)
    col = out // 2
    for bits in NANS[typ]:
        for at, beside in ((5, None), (5, 6), (195, None), (195, 194)):
            d = dy.clone()
            d.view(BITS[typ])[0, at, col] = bits
            if beside is not None:
                d[0, beside, col] = -math.inf if bits < 0 else math.inf
            assert bool(torch.isnan(d[0, at, col]))
            dw, db = torch.empty(1, cols, out, device="cuda"), torch.empty(1, out, device="cuda")
            ctx.weight_gradient(kept, d, dw, db)
            assert bool(torch.isnan(dw[0, :, col]).all()) and math.isnan(float(db[0, col])), hex(bits)
            ok = torch.ones(out, dtype=torch.bool, device="cuda")
            ok[col] = False
            assert torch.equal(dw[..., ok].double(), clean[..., ok])
