"""Angles of rotary positions far out, against whole-number arithmetic: 1e-9 of a turn at any position, of frequencies up to 1e12 radians.

Frequencies are binary64 and so are rational numbers; an angle's turns come from 120 digits of pi.  Bound, u = 2^-24: the angle 2 pi 1e-9, sine and cosine 4 u, a product and the
sum one u each: (6 u + 2 pi 1e-9) (|a| + |b|) + u |out|."""
import math
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PI = Fraction(int("3141592653589793238462643383279502884197169399375105820974944592307816406286208998628034825342117067982148086513282306647"), 10 ** 120)


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2308_09187_amd import qgx as m
    c = m.Context(1024, 1, 256)
    yield c
    c.close()


def angle(position, frequency):
    """position * frequency less whole turns, in radians."""
    turns = position * Fraction(frequency) / (2 * PI)
    return float((turns - round(turns)) * 2 * PI)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("frequencies", [[1.0, 1e-4, 0.37, 0.9999], [777.7, 1e6, -12345.6789, 3e-9], [1e12, -1e12, 9.87654321e11, 2.0 ** 39]])
def test_angles(ctx, frequencies, neighbours, back):
    from paper_2308_09187_amd import qgx
    P = len(frequencies)
    r = qgx.Rotary((P,), frequencies, neighbours)
    positions = [0, 1, -1, (1 << 31) - 1, -(1 << 31), 1 << 24, 123456789, -987654321, 2000000011, 5]
    g = np.random.default_rng(1)
    positions += [int(p) for p in g.integers(-(1 << 31), 1 << 31, 200)]
    x = torch.from_numpy(g.standard_normal((len(positions), 3, 2 * P)).astype(np.float32)).cuda()
    got = ctx.rotary(x, r, torch.tensor([positions], dtype=torch.int32, device="cuda"), back=back).double().cpu().numpy()
    a = np.array([[angle(p, f) for f in frequencies] for p in positions])[:, None] * (-1 if back else 1)
    i = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if neighbours else (slice(0, P), slice(P, 2 * P))
    v = x.double().cpu().numpy()
    size = np.abs(v[..., i[0]]) + np.abs(v[..., i[1]])
    for at, want in ((i[0], v[..., i[0]] * np.cos(a) - v[..., i[1]] * np.sin(a)), (i[1], v[..., i[0]] * np.sin(a) + v[..., i[1]] * np.cos(a))):
        assert (np.abs(got[..., at] - want) <= (6 * U + 2 * math.pi * 1e-9) * size + U * np.abs(want)).all()


def test_the_largest_frequency_is_finite(ctx):
    """A turn of some angle (its digits are not held any more), no NaN; beyond it the rotation is refused before it is made."""
    from paper_2308_09187_amd import qgx
    most = math.ldexp(float.fromhex("0x1.fffffffffffffp+1023"), -31)
    r = qgx.Rotary((2,), [most, -most])
    x = torch.randn(3, 1, 4, device="cuda")
    y = ctx.rotary(x, r, torch.tensor([[-(1 << 31), (1 << 31) - 1, 0]], dtype=torch.int32, device="cuda"))
    assert bool(torch.isfinite(y).all()) and torch.equal(y[2], x[2])
    n = (x[..., :2] ** 2 + x[..., 2:] ** 2)
    assert torch.allclose(y[..., :2] ** 2 + y[..., 2:] ** 2, n, rtol=1e-5)
    r.frequencies[0] = most * 2                            # (past the plan's own check)
    with pytest.raises(qgx.QgxError) as e:
        ctx.rotary(x, r, torch.zeros(1, 3, dtype=torch.int32, device="cuda"))
    assert e.value.status == qgx.ERR_ARG
