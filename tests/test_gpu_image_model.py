"""examples/image_model.py: its gradients, as the kernels leave them in V, against automatic differentiation of the same model in 64 bits; that it runs
through the coded exchange; a captured step.

Bounds.  A weight gradient sum x dy differs from the exact one by what keeping x in 8 bits does, less than a step of each element: sum of step |dy| over the rows,
and by some ten products and sums in a chain over at most 300 terms: 300 2^-24 ten times over, 2e-4 of the sum of magnitudes.  The norm's gradients, of
dz h with h off by less than s = step rstd and |silu'| <= 1.1, |silu''| <= 1/2: |dy| (1.1 s + s |w| (|h| + s) / 2), and |dy| s |w| / 2, summed."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("image_model", os.path.join(ROOT, "examples", "image_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(model, X, embedding, tokens, targets):
    """One worker's loss, gradient [d] and what enters the bounds, in 64 bits on the CPU."""
    X = X.double().cpu().requires_grad_(True)
    p = {n: model.run_of(X, n) for n in model.sizes}
    B, P, D, H, G = *tokens.shape, model.D, model.H, model.G
    x0 = embedding.double().cpu()[tokens].view(B, P, G, D // G)
    mean, var = x0.mean((1, 3), keepdim=True), x0.var((1, 3), unbiased=False, keepdim=True)
    h = ((x0 - mean) / torch.sqrt(var + 1e-5)).view(B, P, D)
    z = h * p["norm_w"] + p["norm_b"]
    x = z * torch.sigmoid(z)
    x.retain_grad()
    freq = torch.tensor(list(model.rotary.frequencies), dtype=torch.float64)
    axis = torch.repeat_interleave(torch.arange(2), torch.tensor(model.rotary.pairs))
    angle = (model.positions.cpu().double()[axis].t() * freq).unsqueeze(1)                # [P, 1, pairs]

    def turn(t):
        t = t.view(B, P, H, D // H)
        a, b = t.chunk(2, -1)
        return torch.cat([a * torch.cos(angle) - b * torch.sin(angle), a * torch.sin(angle) + b * torch.cos(angle)], -1).transpose(1, 2)

    lin = {"wq": x @ p["wq"] + p["bq"], "wk": x @ p["wk"], "wv": x @ p["wv"]}
    for t in lin.values():
        t.retain_grad()
    scores = turn(lin["wq"]) @ turn(lin["wk"]).transpose(-1, -2) / math.sqrt(D // H)
    mixed = (torch.softmax(scores, -1) @ lin["wv"].view(B, P, H, D // H).transpose(1, 2)).transpose(1, 2).reshape(B, P, D)
    lin["head"] = mixed @ p["head"]
    lin["head"].retain_grad()
    loss = torch.nn.functional.cross_entropy(lin["head"].view(B * P, -1), targets.view(-1), ignore_index=-1)
    loss.backward()
    return loss.item(), X.grad, {n: t.grad.reshape(B * P, -1) for n, t in lin.items()}, dict(x=x.detach().reshape(B * P, D), mixed=mixed.detach().reshape(B * P, D), h=h, dx=x.grad)


def steps_of(kept, k, cols):
    return torch.exp2(kept.powers[k].double().cpu() - 127.0).repeat_interleave(32, -1)[..., :cols]


def test_gradients_in_v(example):
    t = example.Trainer(K=3, seed=5)
    m = t.model
    m.run_of(t.X, "norm_b").normal_(generator=t.gen)
    m.run_of(t.X, "norm_w").add_(0.3)
    m.run_of(t.X, "bq").normal_(generator=t.gen)
    tokens, targets = t.data()
    t.V.fill_(7.0)
    loss, kept = m.gradients(t.ctx, t.X, t.V, t.embedding, tokens, targets, 3)
    losses = []
    for k in range(3):
        ref, grad, back, mid = reference(m, t.X, t.embedding, tokens[k].cpu(), targets[k].cpu())
        losses.append(ref)
        run = lambda name: m.run_of(t.V, name)[k].double().cpu()  # noqa: E731
        for name, source, value in (("wq", "kept", "x"), ("wk", "kept", "x"), ("wv", "kept", "x"), ("head", "kept_mixed", "mixed")):
            dy = back[name].abs()
            step = steps_of(kept[source], k, m.D).reshape(-1, m.D)
            bound = step.t() @ dy + 2e-4 * (mid[value].abs().t() @ dy) + 1e-9
            assert ((run(name) - m.run_of(grad, name)).abs() <= bound).all(), name
        assert ((run("bq") - m.run_of(grad, "bq")).abs() <= 2e-4 * back["wq"].abs().sum(0) + 1e-9).all()
        rstd = kept["rstd"][k].double().cpu().repeat_interleave(m.D // m.G, -1)[:, None]
        s = steps_of(kept["kept0"], k, m.D) * rstd
        w, dy, h = m.run_of(t.X, "norm_w").double().cpu().abs(), mid["dx"].abs(), mid["h"].abs()
        assert ((run("norm_w") - m.run_of(grad, "norm_w")).abs() <= (dy * (1.1 * s + 0.5 * s * w * (h + s) + 4e-4 * h)).sum((0, 1)) + 1e-9).all()
        assert ((run("norm_b") - m.run_of(grad, "norm_b")).abs() <= (dy * (0.5 * s * w + 4e-4)).sum((0, 1)) + 1e-9).all()
    assert abs(loss.item() - sum(losses) / 3) < 1e-4 and t.ctx.poll_error() == 0
    t.ctx.close()


def test_it_runs_through_the_exchange(example):
    t = example.Trainer(K=2, seed=1)
    losses = [t.step() for _ in range(6)]
    assert all(math.isfinite(x.item()) for x in losses) and t.ctx.poll_error() == 0 and t.ctx.scalars()["t"] == 7
    assert torch.isfinite(t.X).all()
    t.ctx.close()


def test_the_gradients_replayed_as_a_graph(example):
    """Forward, kept activations and backward of one step captured once; every replay equals the eager step on the same inputs, bit for bit."""
    t = example.Trainer(K=2, seed=2)
    m = t.model
    tokens, targets = t.data()
    V = torch.zeros_like(t.V)
    m.gradients(t.ctx, t.X, V, t.embedding, tokens, targets, 4)       # (libraries make their workspaces)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.gradients(t.ctx, t.X, V, t.embedding, tokens, targets, 4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        m.gradients(t.ctx, t.X, V, t.embedding, tokens, targets, 4)
    for _ in range(3):
        a, b = t.data()
        tokens.copy_(a)
        targets.copy_(b)
        t.X.mul_(1.01)
        m.gradients(t.ctx, t.X, t.V, t.embedding, tokens, targets, 4)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.allclose(V, t.V, rtol=2e-4, atol=1e-7)          # (the library's products may choose another order when captured)
    t.ctx.close()
