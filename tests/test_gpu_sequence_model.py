"""examples/sequence_model.py: its gradients, as the kernels leave them in V, against automatic differentiation of the same model in
64 bits; the clipped vectors; and that it learns.

Bound of the gradients: some ten products and sums in a chain, each over at most 200 terms and so off by at most 200 2^-24 of its
magnitudes: 1.2e-4 of a gradient tensor's largest element, rounded up."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("sequence_model", os.path.join(ROOT, "examples", "sequence_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(model, X, embedding, tokens, targets):
    """One worker's loss and gradient [d], in 64 bits on the CPU."""
    X = X.double().cpu().requires_grad_(True)
    p = {n: model.run_of(X, n) for n in model.sizes}
    x = embedding.double().cpu()[tokens]                               # [B, L, D]
    x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-5) * p["norm_w"] + p["norm_b"]
    B, L, D, H = *x.shape, model.H

    def heads(t):
        return t.view(B, L, H, D // H).transpose(1, 2)

    q, k, v = heads(x @ p["wq"]), heads(x @ p["wk"]), heads(x @ p["wv"])
    distance = torch.arange(L)[:, None] - torch.arange(L)[None, :]
    b = model.buckets
    row = [next(b._rows[i] for i in range(b._c.n) if b._bounds[i] <= -n < b._bounds[i + 1]) for n in range(L)]
    bias = p["table"][torch.tensor(row)[distance.clamp_min(0)]].permute(2, 0, 1)
    scores = (q @ k.transpose(-1, -2) / math.sqrt(D // H) + bias).masked_fill(distance < 0, -math.inf)
    mixed = (torch.softmax(scores, -1) @ v).transpose(1, 2).reshape(B, L, D)
    loss = torch.nn.functional.cross_entropy((mixed @ p["head"]).view(B * L, -1), targets.view(-1), ignore_index=-1)
    loss.backward()
    return loss.item(), X.grad


def test_gradients_in_v(example):
    t = example.Trainer(K=3, seed=5)
    m = t.model
    m.run_of(t.X, "table").normal_(generator=t.gen)
    m.run_of(t.X, "norm_b").normal_(generator=t.gen)
    tokens, targets = t.data()
    loss, g = m.gradients(t.ctx, t.X, t.V, t.embedding, tokens, targets)
    refs = [reference(m, t.X, t.embedding, tokens[k].cpu(), targets[k].cpu()) for k in range(3)]
    assert abs(loss.item() - np.mean([r[0] for r in refs])) < 1e-4
    norms = []
    for k, (_, grad) in enumerate(refs):
        for name in m.sizes:
            got = (g[name][k] if name in g else m.run_of(t.V, name)[k]).double().cpu().reshape(-1)
            want = m.run_of(grad, name).reshape(-1)
            assert (got - want).abs().max() <= 1.3e-4 * want.abs().max(), name
        norms.append(grad.norm().item())
    # clipped into V: every run scaled by the same factor, the norm as it was
    for name, buffer in t.matrices.items():
        buffer.copy_(g[name])
    before = {n: (g[n] if n in g else m.run_of(t.V, n).reshape(3, -1)).clone() for n in m.sizes}
    got = t.ctx.clip_gradients(t.list, 0.5 * min(norms), out=t.V).cpu().numpy()
    assert np.allclose(got, norms, rtol=1e-3)
    for k in range(3):
        for n in m.sizes:
            want = before[n][k] * (0.5 * min(norms) / float(got[k]))
            assert torch.allclose(m.run_of(t.V, n)[k].reshape(-1), want, rtol=1e-5, atol=1e-12)
    t.ctx.close()


def test_it_learns(example):
    t = example.Trainer(K=2, seed=1)
    losses = [t.step() for _ in range(60)]
    losses = [x.item() for x in losses]
    assert losses[0] > 2.0 and losses[-1] < 0.3 and t.ctx.poll_error() == 0
    t.ctx.close()
