"""Cases for the operators between a model's backward pass and the dual vectors V [K][d] of the coded exchange.

Three operators, all with parameters in the iterate X [d] and gradients in the K workers' rows of V:
  clip   each worker's global gradient norm over its many tensors, and the clipped tensors gathered into V
  norm   layer norm, forward, and backward with the parameters' gradients reduced per worker
  bias   the learned relative position bias by buckets, added to attention scores, and its gradient per worker

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is true, through the framework's
entry points; ``exact`` has their definitions in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}

# The GAN-shaped layout of the benchmark: 14 tensors, weights and bias vectors.
GAN = (1048576, 8192, 2097152, 256, 524288, 128, 73728, 64, 73728, 524288, 2097152, 2359296, 512, 1048576)


def listed():
    return [
        # Clipping before the coded exchange.  A small game's vectors (the benchmark's 4 x 2^16), where the launches count.
        dict(name="clip_small", op="clip", K=4, tensors=1, d=1 << 16, layout=0, type="f32", norm="l2"),
        # A mixed-precision GAN: weight matrices in bfloat16, vectors in binary32, 14 tensors for each of 8 workers.
        dict(name="clip_gan", op="clip", K=8, tensors=14, d=sum(GAN), layout=-1, type="mixed", norm="l2"),
        # A model of 16.8 M parameters in 150 tensors of every size, odd ones among them, eight workers.
        dict(name="clip_tensors", op="clip", K=8, tensors=150, d=1 << 24, layout=5, type="f32", norm="l2"),
        # The benchmark's largest batch, 16 x 2^26: far beyond any cache.
        dict(name="clip_large", op="clip", K=16, tensors=1, d=1 << 26, layout=0, type="f32", norm="l2"),
        # Layer norm.  One token of a sequence that is being generated: latency alone.
        dict(name="norm_token", op="norm", back=False, K=1, rows=1, cols=1024, type="bf16"),
        # A training batch's activations, eight workers.
        dict(name="norm_rows", op="norm", back=False, K=8, rows=4096, cols=4096, type="bf16"),
        # Backward with an odd width and an odd number of rows, in binary32: small images' patches.
        dict(name="norm_grad_odd", op="norm", back=True, K=4, rows=197, cols=1001, type="f32"),
        # Backward of a training batch.
        dict(name="norm_grad_rows", op="norm", back=True, K=8, rows=4096, cols=2048, type="bf16"),
        # Position bias.  The next token of 32 sequences of different lengths against their keys.
        dict(name="bias_token", op="bias", back=False, K=1, batch=32, heads=16, q=1, k=4099, table=32, far=128,
             causal=True, scores=True, ragged=True, type="bf16"),
        # Scores of a training batch, both directions visible.
        dict(name="bias_scores", op="bias", back=False, K=1, batch=8, heads=16, q=1024, k=1024, table=32, far=128,
             causal=False, scores=True, ragged=False, type="bf16"),
        # Gradient for small images' patches: an odd length, binary32, both directions.
        dict(name="bias_grad_odd", op="bias", back=True, K=4, batch=3, heads=6, q=197, k=197, table=32, far=64,
             causal=False, scores=True, ragged=False, type="f32"),
        # Gradient of a causal training batch, eight workers.
        dict(name="bias_grad_causal", op="bias", back=True, K=8, batch=2, heads=16, q=1024, k=1024, table=32, far=128,
             causal=True, scores=True, ragged=False, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["clip", "norm", "bias"])
    if op == "clip":
        K = _log_int(rng, 1, 16)
        d = _log_int(rng, 1 << 8, 1 << 26)
        tensors = min(_log_int(rng, 1, 300), d // 8)
        return dict(op=op, K=K, tensors=tensors, d=d, layout=rng.randrange(1, 1000),
                    type=rng.choice(["f32", "f32", "bf16", "f16", "mixed"]), norm=rng.choice(["l2", "l2", "l2", "linf"]))
    if op == "norm":
        back = rng.random() < 0.6
        K, cols = _log_int(rng, 1, 8), _log_int(rng, 8, 16384)
        rows = _log_int(rng, 1, max(1, min(8192, (1 << 27) // (K * cols))))
        return dict(op=op, back=back, K=K, rows=rows, cols=cols, type=rng.choice(["f32", "bf16", "bf16", "f16"]))
    back = rng.random() < 0.5
    kind = rng.choice(["token", "square", "square", "cross"])
    heads, table, far = rng.randrange(1, 25), rng.choice([8, 16, 32, 64]), rng.choice([64, 128, 250])
    typ, causal = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.random() < 0.5
    if kind == "token" and not back:
        q, k, batch = 1, _log_int(rng, 16, 32768), _log_int(rng, 1, 64)
        return dict(op=op, back=False, K=1, batch=batch, heads=heads, q=q, k=k, table=table, far=far, causal=True,
                    scores=True, ragged=True, type=typ)
    q = _log_int(rng, 16, 2048)
    k = q if kind != "cross" else _log_int(rng, 16, 2048)
    K = _log_int(rng, 1, 8) if back else 1
    batch = _log_int(rng, 1, max(1, min(16, (1 << 28) // (K * heads * q * k))))
    return dict(op=op, back=back, K=K, batch=batch, heads=heads, q=q, k=k, table=table, far=far, causal=causal,
                scores=back or rng.random() < 0.8, ragged=False, type=typ)


def _up4(n):
    return (n + 3) // 4 * 4


def _tensor_sizes(case):
    """Elements of every tensor: the GAN's, one of d, or a cut of d with sizes over several orders of magnitude."""
    if case["layout"] < 0:
        return list(GAN)
    if case["tensors"] == 1:
        return [case["d"]]
    rng = random.Random(case["layout"])
    weights = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["tensors"])]
    total = sum(weights)
    return [max(1, int(case["d"] * w / total)) for w in weights]


def _tensor_types(case, sizes):
    if case["type"] != "mixed":
        return [case["type"]] * len(sizes)
    return ["bf16" if n > 10000 else "f32" for n in sizes]


def _offsets(sizes):
    off, at = [], 0
    for n in sizes:
        off.append(at)
        at += _up4(n)
    return off, at


def bucket_bounds(case):
    """Buckets of the relative position delta = key - query: bounds (ascending) and the table row of each interval.

    m buckets a side: distances below e = m // 2 have one each, further ones are spaced by their logarithm up to `far`:
    bucket e + t starts at the smallest n with n >= e (far / e)^(t / (m - e)).  Causal: keys after the query are in none."""
    m = case["table"] if case["causal"] else case["table"] // 2
    e = m // 2
    r = m - e
    lo = list(range(e))
    for t in range(r):
        n = max(e, 1)
        while n ** r < e ** (r - t) * case["far"] ** t:
            n += 1
        lo.append(max(n, lo[-1] + 1) if lo else n)
    bounds, rows = [-(1 << 30)], []
    for b in range(m - 1, -1, -1):                    # keys before the query, the furthest first
        bounds.append(1 - lo[b])
        rows.append(b)
    if not case["causal"]:
        for b in range(m):
            end = lo[b + 1] if b + 1 < m else 1 << 30
            if end > 1:                               # distance 0 belongs to the other side
                bounds.append(end)
                rows.append(m + b)
    return bounds, rows


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _prepare_clip(case, gen):
    sizes = _tensor_sizes(case)
    types = _tensor_types(case, sizes)
    off, d = _offsets(sizes)
    K = case["K"]
    # a scale per tensor and per worker, as gradients have them
    tscale = (10.0 ** (-4.0 + 2.0 * torch.rand(len(sizes), generator=gen, device="cuda"))).tolist()
    wscale = torch.exp(_normal(gen, K, 1))
    tensors, total = [], torch.zeros(K, device="cuda")
    for n, t, s in zip(sizes, types, tscale):
        x = _normal(gen, K, n).mul_(wscale).mul_(s).to(TYPES[t])
        tensors.append(x)
        f = x.float()
        total = total + (f * f).sum(1) if case["norm"] == "l2" else torch.maximum(total, f.abs().amax(1))
        del f
    norms = total.sqrt() if case["norm"] == "l2" else total
    # about half the workers exceed it; a single one does
    limit = float(norms.median()) * 0.75
    V = torch.zeros(K, d, device="cuda")
    state = dict(case=case, tensors=tensors, off=off, V=V, limit=limit)
    if own:
        from paper_2308_09187_amd import qgx
        state["ctx"] = qgx.Context(d, K, 8192)
        state["list"] = state["ctx"].tensor_list(tensors, off)
        state["kind"] = qgx.NORM_L2 if case["norm"] == "l2" else qgx.NORM_LINF
    return state


def _prepare_norm(case, gen):
    K, rows, cols, typ = case["K"], case["rows"], case["cols"], TYPES[case["type"]]
    # activations: every row has an offset and a scale, some channels are larger
    x = _normal(gen, K, rows, cols)
    x = x * torch.exp(0.5 * _normal(gen, K, rows, 1)) + 0.5 * _normal(gen, K, rows, 1) + _normal(gen, cols)
    x = x.to(typ)
    d = 8 + 2 * _up4(cols)
    X = torch.zeros(d, device="cuda")
    w, b = X[8:8 + cols], X[8 + _up4(cols):8 + _up4(cols) + cols]
    w.copy_(1.0 + 0.2 * _normal(gen, cols))
    b.copy_(0.1 * _normal(gen, cols))
    state = dict(case=case, x=x, w=w, b=b, eps=1e-5)
    if case["back"]:
        f = x.float()
        mean = f.mean(2)
        f = f - mean.unsqueeze(2)
        rstd = 1.0 / torch.sqrt((f * f).mean(2) + 1e-5)
        del f
        V = torch.zeros(K, d, device="cuda")
        state.update(dy=(1e-2 * _normal(gen, K, rows, cols)).to(typ), mean=mean, rstd=rstd,
                     dw=V[:, 8:8 + cols], db=V[:, 8 + _up4(cols):8 + _up4(cols) + cols])
    if own:
        from paper_2308_09187_amd import qgx
        state["ctx"] = qgx.Context(d, K, 4096)
    return state


def _prepare_bias(case, gen):
    K, n, h, q, k, typ = (case["K"], case["batch"], case["heads"], case["q"], case["k"], TYPES[case["type"]])
    bounds, rows = bucket_bounds(case)
    R = case["table"]
    d = 8 + _up4(R * h)
    X = torch.zeros(d, device="cuda")
    table = X[8:8 + R * h].view(R, h)
    table.copy_(_normal(gen, R, h))
    state = dict(case=case, bounds=bounds, rows=rows, table=table, positions=None, offset=0)
    if case["ragged"]:
        # sequences of different lengths: the query's position, the longest with all keys before it
        state["positions"] = torch.randint(0, k, (n,), generator=gen, device="cuda").to(torch.int32)
    elif case["causal"] and k > q:
        state["offset"] = k - q                       # the last q positions of k
    if case["back"]:
        V = torch.zeros(K, d, device="cuda")
        state["ds"] = (1e-2 * _normal(gen, K, n, h, q, k)).to(typ)
        state["dtable"] = V[:, 8:8 + R * h].unflatten(1, (R, h))
    elif case["scores"]:
        state["scores"] = (2.0 * _normal(gen, n, h, q, k)).to(typ)
    else:
        state["scores"] = None
    if own:
        from paper_2308_09187_amd import qgx
        state["ctx"] = qgx.Context(d, K, 4096)
        state["buckets"] = qgx.Buckets(bounds, rows)
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    return {"clip": _prepare_clip, "norm": _prepare_norm, "bias": _prepare_bias}[case["op"]](case, gen)


# -- the plain forms --------------------------------------------------------------------------------------------------


def _plain_clip(s):
    total = torch.zeros(s["case"]["K"], device="cuda")
    for t in s["tensors"]:
        x = t.float()
        if s["case"]["norm"] == "l2":
            total = total + (x * x).sum(1)
        else:
            total = torch.maximum(total, x.abs().amax(1))
    norms = total.sqrt() if s["case"]["norm"] == "l2" else total
    clip = torch.isfinite(norms) & (norms > s["limit"])
    coef = torch.where(clip, s["limit"] / norms, torch.ones_like(norms)).unsqueeze(1)
    for t, off in zip(s["tensors"], s["off"]):
        s["V"][:, off:off + t.shape[1]] = t.float() * coef
    return {"V": s["V"], "norms": norms}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(2, keepdim=True)
    x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).mean(2, keepdim=True) + s["eps"])
    y = (x * rstd * s["w"] + s["b"]).to(s["x"].dtype)
    return {"y": y, "mean": mean.squeeze(2), "rstd": rstd.squeeze(2)}


def _plain_norm_back(s):
    rstd = s["rstd"].unsqueeze(2)
    h = (s["x"].float() - s["mean"].unsqueeze(2)) * rstd
    dy = s["dy"].float()
    s["dw"].copy_((dy * h).sum(1))
    s["db"].copy_(dy.sum(1))
    g = dy * s["w"]
    dx = rstd * (g - g.mean(2, keepdim=True) - h * (g * h).mean(2, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dw": s["dw"], "db": s["db"]}


def _intervals(s, delta):
    """Index of the interval of every delta, and whether there is one."""
    bounds = torch.tensor(s["bounds"], device="cuda", dtype=torch.int64)
    at = torch.bucketize(delta, bounds, right=True) - 1
    seen = (at >= 0) & (at < len(s["rows"]))
    return at.clamp(0, len(s["rows"]) - 1), seen


def _plain_bias(s):
    c = s["case"]
    i = torch.arange(c["q"], device="cuda").view(-1, 1)
    j = torch.arange(c["k"], device="cuda").view(1, -1)
    delta = j - i - s["offset"]
    if s["positions"] is not None:
        delta = delta.unsqueeze(0) - s["positions"].to(torch.int64).view(-1, 1, 1)     # [n, q, k]
    at, seen = _intervals(s, delta)
    rows = torch.tensor(s["rows"], device="cuda", dtype=torch.int64)[at]
    bias = torch.movedim(s["table"][rows], -1, -3)                                     # [.., h, q, k]
    out = bias if s["scores"] is None else s["scores"].float() + bias
    seen = seen.unsqueeze(-3)
    return {"out": torch.where(seen, out, torch.full_like(out, -math.inf)).to(TYPES[c["type"]])}


def _plain_bias_back(s):
    c = s["case"]
    q, k = c["q"], c["k"]
    x = s["ds"].float().sum(1).flip(-2)                    # [K, h, q, k], queries from the last to the first
    # one more entry than columns in every row but the last shifts row r by r: the columns are then the diagonals
    w = q + k - 1
    x = torch.nn.functional.pad(x, (0, q)).flatten(-2)[..., :q * w].unflatten(-1, (q, w)).sum(-2)   # [K, h, q + k - 1]
    at, seen = _intervals(s, torch.arange(w, device="cuda") - (q - 1) - s["offset"])
    rows = torch.tensor(s["rows"], device="cuda", dtype=torch.int64)[at]
    hot = (rows.unsqueeze(0) == torch.arange(c["table"], device="cuda").view(-1, 1)) & seen         # [R, w]
    x = torch.where(seen, x, torch.zeros_like(x))
    for r in range(c["table"]):
        s["dtable"][:, r].copy_((x * hot[r]).sum(-1))
    return {"dtable": s["dtable"]}


def run(state):
    case = state["case"]
    if not own:
        if case["op"] == "clip":
            return _plain_clip(state)
        if case["op"] == "norm":
            return _plain_norm_back(state) if case["back"] else _plain_norm(state)
        return _plain_bias_back(state) if case["back"] else _plain_bias(state)
    ctx = state["ctx"]
    if case["op"] == "clip":
        norms = ctx.clip_gradients(state["list"], state["limit"], norm=state["kind"], out=state["V"])
        return {"V": state["V"], "norms": norms}
    if case["op"] == "norm":
        if not case["back"]:
            y, mean, rstd = ctx.layer_norm(state["x"], state["w"], state["b"], state["eps"])
            return {"y": y, "mean": mean, "rstd": rstd}
        dx = ctx.layer_norm_backward(state["dy"], state["x"], state["w"], state["mean"], state["rstd"],
                                     dw=state["dw"], db=state["db"])
        return {"dx": dx, "dw": state["dw"], "db": state["db"]}
    if not case["back"]:
        if state["scores"] is None:
            out = ctx.position_bias(state["table"], state["buckets"], case["q"], case["k"], dtype=TYPES[case["type"]],
                                    q_offset=state["offset"])
        else:
            out = ctx.add_position_bias(state["scores"], state["table"], state["buckets"], q_offset=state["offset"],
                                        positions=state["positions"])
        return {"out": out}
    ctx.position_bias_backward(state["ds"], state["buckets"], state["dtable"], q_offset=state["offset"])
    return {"dtable": state["dtable"]}


# -- what a pass cannot do without ------------------------------------------------------------------------------------


def _visible(case):
    """(query, key) pairs that lie in a bucket, of q * k; positions of ragged sequences are taken at their mean."""
    q, k = case["q"], case["k"]
    if not case["causal"]:
        return q * k
    if case["ragged"]:
        return q * (k + 1) // 2
    p = max(0, k - q)
    return sum(min(k, i + p + 1) for i in range(q))


def work(case):
    if case["op"] == "clip":
        sizes = _tensor_sizes(case)
        read = sum(n * SIZE[t] for n, t in zip(sizes, _tensor_types(case, sizes)))
        return {"bytes": case["K"] * (read + 4 * sum(sizes)), "flops": 3 * case["K"] * sum(sizes)}
    if case["op"] == "norm":
        n, rows = case["K"] * case["rows"] * case["cols"], case["K"] * case["rows"]
        if not case["back"]:
            return {"bytes": 2 * n * SIZE[case["type"]] + 8 * rows + 8 * case["cols"], "flops": 8 * n}
        return {"bytes": 3 * n * SIZE[case["type"]] + 8 * rows + 4 * case["cols"] * (1 + 2 * case["K"]), "flops": 14 * n}
    size, heads = SIZE[case["type"]], case["K"] * case["batch"] * case["heads"]
    seen = _visible(case)
    table = 4 * case["table"] * case["heads"]
    if case["back"]:
        return {"bytes": heads * seen * size + case["K"] * table, "flops": heads * seen}
    if not case["scores"]:
        return {"bytes": case["heads"] * case["q"] * case["k"] * size + table, "flops": 0}
    return {"bytes": heads * (seen + case["q"] * case["k"]) * size + table, "flops": heads * seen}


# -- the definitions in 64 bits ---------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        V = torch.zeros(s["V"].shape, dtype=torch.float64, device="cuda")
        for t, off in zip(s["tensors"], s["off"]):
            V[:, off:off + t.shape[1]] = t
        p = 2.0 if case["norm"] == "l2" else math.inf
        norms = torch.stack([torch.linalg.vector_norm(V[k], p) for k in range(case["K"])])
        for k, n in enumerate(norms.tolist()):
            if n > s["limit"] and math.isfinite(n):
                V[k] *= s["limit"] / n
        return {"V": V, "norms": norms}
    if case["op"] == "norm":
        return _exact_norm(case, s)
    return _exact_bias(case, s)


def _exact_norm(case, s):
    w, b, n = s["w"].double(), s["b"].double(), case["cols"]
    out = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
    if not case["back"]:
        mean = torch.empty(s["x"].shape[:2], dtype=torch.float64, device="cuda")
        rstd = torch.empty_like(mean)
        for k in range(case["K"]):
            x = s["x"][k].double()
            var, mu = torch.var_mean(x, dim=1, unbiased=False)
            mean[k], rstd[k] = mu, torch.rsqrt(var + s["eps"])
            out[k] = torch.addcmul(b, (x - mu[:, None]) * rstd[k][:, None], w)
        return {"y": out, "mean": mean, "rstd": rstd}
    dw = torch.empty(case["K"], n, dtype=torch.float64, device="cuda")
    db = torch.empty_like(dw)
    for k in range(case["K"]):
        r = s["rstd"][k].double()[:, None]
        h = (s["x"][k].double() - s["mean"][k].double()[:, None]) * r
        dy = s["dy"][k].double()
        dw[k], db[k] = torch.sum(dy * h, dim=0), torch.sum(dy, dim=0)
        # dx = r (I - 1 1^T / n - h h^T / n) (w dy), row by row
        g = dy * w
        a1, a2 = torch.sum(g, 1, keepdim=True) / n, torch.sum(g * h, 1, keepdim=True) / n
        out[k] = (g - a1 - h * a2) * r
    return {"dx": out, "dw": dw, "db": db}


def _exact_bias(case, s):
    bounds, rows, q, k = s["bounds"], s["rows"], case["q"], case["k"]
    lo = -(q + k + max(s["offset"], k))
    hi = q + k
    row_of = np.full(hi - lo + 1, -1, np.int64)            # of delta - lo, -1: in no bucket
    for b, r in enumerate(rows):
        first, last = max(bounds[b], lo), min(bounds[b + 1] - 1, hi)
        if first <= last:
            row_of[first - lo:last - lo + 1] = r
    if case["back"]:
        out = torch.zeros(case["K"], case["table"], case["heads"], dtype=torch.float64, device="cuda")
        ds = torch.zeros(case["K"], case["heads"], q, k, dtype=torch.float64, device="cuda")
        for n in range(case["batch"]):
            ds += s["ds"][:, n]
        for diag in range(-(q - 1), k):
            r = int(row_of[diag - s["offset"] - lo])
            if r >= 0:
                out[:, r] += torch.diagonal(ds, diag, -2, -1).sum(-1)
        return {"dtable": out}
    table = s["table"].double()
    padded = torch.cat([table, torch.full((1, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")])
    row_t = torch.from_numpy(row_of).cuda()

    def bias_at(position):
        i = torch.arange(q, device="cuda")[:, None] + position
        j = torch.arange(k, device="cuda")[None, :]
        return padded[row_t[j - i - lo]].permute(2, 0, 1)

    if s["positions"] is None:
        bias = bias_at(s["offset"])
        return {"out": bias if s["scores"] is None else s["scores"].double() + bias}
    return {"out": torch.stack([s["scores"][n].double() + bias_at(int(p)) for n, p in enumerate(s["positions"].tolist())])}
