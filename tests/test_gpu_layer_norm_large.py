"""Layer norm of many rows: the forms with two rows to a group, which launches take from eight workgroups a compute unit on, in every number of
threads to a row; and the parameters' gradients without dx where the workgroups' sums go through scratch.

The order of a row's sums does not depend on how many rows a group takes, so the rows have to come out as they do in calls of few rows, bit
for bit; some of them are held against the formulas in 64 bits as well (bounds: test_gpu_layer_norm.py)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_layer_norm import back_inputs, check_backward, check_forward, ctx, host, put, rnd  # noqa: E402, F401

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# threads to a row and pieces to a thread, columns of binary32
FORMS = {(4, 1): 13, (4, 2): 29, (16, 1): 50, (16, 2): 101, (64, 1): 203, (64, 2): 450, (64, 3): 701, (256, 1): 1001, (256, 2): 1903}


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("form", list(FORMS), ids=str)
def test_two_rows_to_a_group(ctx, form, typ):  # noqa: F811
    lanes, _ = form
    cols = FORMS[form] * (1 if typ == "f32" else 2)            # (and odd in binary32)
    if typ != "f32":
        cols -= 3
    groups, K = max(1, 256 // lanes), 3
    few = 8 * torch.cuda.get_device_properties(0).multi_processor_count * groups          # below twice as many rows one is taken at a time
    rows = (2 * few // K + 1) | 1                              # K rows is odd: the last group has one row
    assert rows * K >= 2 * few and rows * K % 2 == 1
    g = torch.Generator(device="cuda")
    g.manual_seed(lanes + cols)
    wide = torch.randn(K, rows, cols + 2, generator=g, device="cuda").mul_(2.0).add_(0.5).to(TYPES[typ])
    x = wide[..., 1:1 + cols]
    w, b = put(1 + 0.3 * rnd(2, cols), "f32"), put(0.5 * rnd(3, cols), "f32")
    y, mean, rstd = ctx.layer_norm(x, w, b)
    for k in range(K):
        for at in range(0, rows, few):
            y1, m1, r1 = ctx.layer_norm(x[k, at:at + few], w, b)
            assert torch.equal(y[k, at:at + few], y1) and torch.equal(mean[k, at:at + few], m1) and torch.equal(rstd[k, at:at + few], r1)
    some = sorted({0, 1, rows - 2, rows - 1, *np.random.default_rng(cols).integers(0, rows, 40).tolist()})
    check_forward(host(x[:, some]), host(w), host(b), float(np.float32(1e-5)), typ, host(y[:, some]), host(mean[:, some]), host(rstd[:, some]))
    left, right = wide[..., 0].clone(), wide[..., -1].clone()
    ctx.layer_norm(x, w, b, out=x)
    assert torch.equal(x, y) and torch.equal(wide[..., 0], left) and torch.equal(wide[..., -1], right)


@pytest.mark.parametrize("typ", list(TYPES))
@pytest.mark.parametrize("K,rows,cols", [(1, 5000, 3), (1, 3001, 24), (2, 1500, 60), (1, 2000, 260), (2, 1500, 1024), (3, 601, 2050), (1, 700, 9000), (1, 300, 16384),
                                         (2, 40, 20001)])
def test_parameters_without_dx(ctx, K, rows, cols, typ):  # noqa: F811
    x, dy, w, mean, rstd = back_inputs(K, rows, cols, typ, seed=7)
    both = [torch.empty(K, cols, device="cuda") for _ in range(2)]
    ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=both[0], db=both[1])
    check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, None, host(both[0]), host(both[1]))
    for which in ((True, False), (False, True), (True, True)):
        got = [torch.full((K, cols), 9.0, device="cuda") if want else None for want in which]
        for weight in (w, None):                               # (they do not depend on the weight)
            assert ctx.layer_norm_backward(dy, x, weight, mean, rstd, dw=got[0], db=got[1], need_dx=False) is None
            assert all(t is None or torch.equal(t, u) for t, u in zip(got, both))
        dx = ctx.layer_norm_backward(dy, x, w, mean, rstd, dw=got[0], db=got[1])
        assert all(t is None or torch.equal(t, u) for t, u in zip(got, both))
        check_backward(host(dy), host(x), host(w), host(mean), host(rstd), typ, host(dx), None, None)
