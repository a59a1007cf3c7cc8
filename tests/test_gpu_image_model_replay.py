"""examples/image_model.py captured: what the framework's own kernels leave is the eager step's, bit for bit, and every tensor it keeps has draws of its own.

(The products in between are a library's, which may choose another order when captured: what comes after them is made again by eager calls from the replay's own inputs.)"""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("image_model_replayed", os.path.join(ROOT, "examples", "image_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_replays_bit_for_bit(example):
    t = example.Trainer(K=2, seed=3)
    m, c = t.model, t.ctx
    tokens, targets = t.data()
    V = torch.zeros_like(t.V)
    side = torch.cuda.Stream()
    m.gradients(c, t.X, V, t.embedding, tokens, targets, 4)           # (libraries make their workspaces)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.gradients(c, t.X, V, t.embedding, tokens, targets, 4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        _, got = m.gradients(c, t.X, V, t.embedding, tokens, targets, 4)
    for _ in range(3):
        a, b = t.data()
        tokens.copy_(a)
        targets.copy_(b)
        t.X.mul_(1.01)
        V.fill_(7.0)
        _, want = m.gradients(c, t.X, t.V, t.embedding, tokens, targets, 4)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for name in ("mean", "rstd"):
            assert torch.equal(got[name], want[name])
        for name in ("kept0", "kept"):
            assert torch.equal(got[name].codes, want[name].codes) and torch.equal(got[name].powers, want[name].powers)
        for name, source, dy, bias in (("wq", "kept", "dq", "bq"), ("wk", "kept", "dk", None), ("wv", "kept", "dv", None), ("head", "kept_mixed", "dlogits", None)):
            db = torch.empty_like(m.run_of(V, bias)) if bias else None
            dw = c.weight_gradient(got[source], got[dy], torch.empty_like(m.run_of(V, name), memory_format=torch.contiguous_format), db)
            assert torch.equal(dw, m.run_of(V, name)) and (db is None or torch.equal(db, m.run_of(V, bias)))
        dw, db = torch.empty_like(m.run_of(V, "norm_w")), torch.empty_like(m.run_of(V, "norm_b"))
        p = {n: m.run_of(t.X, n) for n in m.sizes}
        c.group_norm_backward(got["dx"].view(want["kept0"].shape), got["kept0"], m.G, p["norm_w"], p["norm_b"], got["mean"], got["rstd"], "silu", dw=dw, db=db, need_dx=False)
        assert torch.equal(dw, m.run_of(V, "norm_w")) and torch.equal(db, m.run_of(V, "norm_b"))
    assert c.poll_error() == 0
    c.close()


def test_every_kept_tensor_has_its_own_draws(example):
    t = example.Trainer(K=2, seed=4)
    tokens, targets = t.data()
    _, kept = t.model.gradients(t.ctx, t.X, t.V, t.embedding, tokens, targets, 1)
    assert len({kept[name].tensor for name in ("kept0", "kept", "kept_mixed")}) == 3
    t.ctx.close()
