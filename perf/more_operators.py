"""Cases for the operators of an image or video model's block, trained through the coded exchange.

Four families; parameters are runs of the iterate X [d], their gradients of the K workers' rows of V [K][d]:
  norm   group norm with an activation, channels last: forward, backward, and a training step whose backward pass works from the
         input as it was kept in 8 bits
  keep   activations kept in 8 bits (blocks of 32 with a power of two each, rounded to nearest or without bias) and restored
  grad   the weight gradient of a linear layer, from its kept input, on the matrix cores
  turn   rotary positions with several axes, forward and backward

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is true, through the framework's
entry points; ``exact`` has their definitions in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 32                                                 # elements that share a power of two


def listed():
    return [
        # Group norm.  The smallest feature map of one image that is being generated: latency alone.
        dict(name="norm_image", op="norm", mode="forward", K=1, batch=1, places=64, channels=512, groups=32, act="silu", type="bf16"),
        # Large feature maps, 256 x 256, of a few images: a group's values do not fit a workgroup.
        dict(name="norm_wide", op="norm", mode="forward", K=1, batch=4, places=65536, channels=128, groups=32, act="silu", type="bf16"),
        # A training step of eight workers on 32 x 32 feature maps: forward, the input kept in 8 bits, backward from that.
        dict(name="norm_step", op="norm", mode="step", K=8, batch=16, places=1024, channels=256, groups=32, act="silu", type="bf16"),
        # Backward in binary32 at odd sizes: 13 x 17 places, groups of 15 channels, a leaky unit as a discriminator has it.
        dict(name="norm_grad_odd", op="norm", mode="backward", K=4, batch=3, places=221, channels=90, groups=6, act="leaky", type="f32"),
        # Activations kept and restored.  A training batch, rounded without bias.
        dict(name="keep_rows", op="keep", K=8, rows=4096, cols=2048, unbiased=True, type="bf16"),
        # Small images' patches in binary32, an odd width, rounded to nearest.
        dict(name="keep_odd", op="keep", K=4, rows=197, cols=1001, unbiased=False, type="f32"),
        # Weight gradient.  A small layer of a small batch: latency.
        dict(name="grad_small", op="grad", K=1, rows=64, cols=64, out=64, bias=True, type="bf16"),
        # A training batch of eight workers through a wide layer.
        dict(name="grad_rows", op="grad", K=8, rows=4096, cols=1024, out=4096, bias=True, type="bf16"),
        # Long activations and narrow layers in binary32 (feature maps as rows): few results, each a sum over 65536 rows.
        dict(name="grad_long", op="grad", K=4, rows=65536, cols=256, out=320, bias=True, type="f32"),
        # Rotary positions.  The next token of 32 sequences of different lengths, three axes, far positions.
        dict(name="turn_token", op="turn", back=False, K=1, batch=32, tokens=1, heads=16, dim=128, rest=0, axes=3, neighbours=False, own_positions=True,
             type="bf16"),
        # A video batch: 16 frames of 32 x 32 tokens.
        dict(name="turn_video", op="turn", back=False, K=1, batch=4, tokens=16384, heads=16, dim=128, rest=0, axes=3, neighbours=False, own_positions=False,
             type="bf16"),
        # Backward for small images' patches, four workers, two axes, neighbouring pairs, a part of every head left as it is.
        dict(name="turn_grad", op="turn", back=True, K=4, batch=3, tokens=197, heads=6, dim=80, rest=16, axes=2, neighbours=True, own_positions=False,
             type="f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "keep", "grad", "grad", "turn"])
    typ = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "norm":
        groups, per = rng.choice([1, 4, 6, 8, 16, 32, 32]), _log_int(rng, 2, 40)
        K, batch = _log_int(rng, 1, 8), _log_int(rng, 1, 16)
        places = _log_int(rng, 4, max(4, min(65536, (1 << 25) // (K * batch * groups * per))))
        mode = rng.choice(["forward", "backward", "step"])
        # (the leaky unit's derivative jumps at 0: where a pass makes the statistics itself, their last bits would decide it)
        return dict(op=op, mode=mode, K=K, batch=batch, places=places, channels=groups * per, groups=groups,
                    act=rng.choice(["silu", "silu", "none" if mode == "step" else "leaky", "none"]), type=typ)
    if op == "keep":
        K, cols = _log_int(rng, 1, 8), _log_int(rng, 8, 16384)
        rows = _log_int(rng, 1, max(1, min(16384, (1 << 26) // (K * cols))))
        return dict(op=op, K=K, rows=rows, cols=cols, unbiased=rng.random() < 0.6, type=typ)
    if op == "grad":
        K, cols, out = _log_int(rng, 1, 8), _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        rows = _log_int(rng, 16, max(16, min(65536, (1 << 36) // (K * cols * out), (1 << 28) // (K * max(cols, out)))))
        return dict(op=op, K=K, rows=rows, cols=cols, out=out, bias=rng.random() < 0.7, type=typ)
    K, heads, dim = _log_int(rng, 1, 4), rng.randrange(1, 25), 2 * rng.randrange(16, 97)
    axes = rng.randrange(1, 4)
    tokens = _log_int(rng, 1, 16384)
    batch = _log_int(rng, 1, max(1, min(64, (1 << 27) // (K * heads * dim * tokens))))
    return dict(op=op, back=rng.random() < 0.5, K=K, batch=batch, tokens=tokens, heads=heads, dim=dim, rest=2 * rng.randrange(0, 5), axes=axes,
                neighbours=rng.random() < 0.5, own_positions=rng.random() < 0.5, type=typ)


def _up4(n):
    return (n + 3) // 4 * 4


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


# -- inputs -------------------------------------------------------------------------------------------------------------


def _activations(gen, lead, cols, typ):
    """Rows with a scale and an offset each, some channels larger, as layers make them."""
    ones = (1,) * (len(lead) - 1)
    x = _normal(gen, *lead, cols) * torch.exp(0.4 * _normal(gen, lead[0], *ones, 1))
    return (x * torch.exp(0.5 * _normal(gen, cols)) + _normal(gen, cols)).to(TYPES[typ])


def _prepare_norm(case, gen, state):
    K, N, P, C, G = case["K"], case["batch"], case["places"], case["channels"], case["groups"]
    x = _activations(gen, (K, N, P), C, case["type"])
    d = 8 + 2 * _up4(C)
    X = torch.zeros(d, device="cuda")
    w, b = X[8:8 + C], X[8 + _up4(C):8 + _up4(C) + C]
    w.copy_(1.0 + 0.2 * _normal(gen, C))
    b.copy_(0.3 * _normal(gen, C))
    state.update(x=x, w=w, b=b, eps=1e-5, slope=0.2, d=d)
    if case["mode"] != "forward":
        V = torch.zeros(K, d, device="cuda")
        state.update(dy=(1e-2 * _normal(gen, K, N, P, C)).to(x.dtype), dw=V[:, 8:8 + C], db=V[:, 8 + _up4(C):8 + _up4(C) + C])
    if case["mode"] == "backward":
        f = x.float().view(K, N, P, G, C // G)
        mean = f.mean((2, 4))
        f = f - mean.view(K, N, 1, G, 1)
        state.update(mean=mean, rstd=1.0 / torch.sqrt((f * f).mean((2, 4)) + 1e-5))


def _prepare_keep(case, gen, state):
    state.update(x=_activations(gen, (case["K"], case["rows"]), case["cols"], case["type"]), d=64)


def _prepare_grad(case, gen, state):
    K, R, I, O = case["K"], case["rows"], case["cols"], case["out"]
    # kept after a unit that leaves half of it near zero
    x = _activations(gen, (K, R), I, "f32")
    codes, powers = _keep(x * torch.sigmoid(2.0 * x), None, 0)
    d = 8 + _up4(I * O) + _up4(O)
    V = torch.zeros(K, d, device="cuda")
    at = 8 + _up4(I * O)
    state.update(codes=codes, powers=powers, dy=(1e-3 * _normal(gen, K, R, O)).to(TYPES[case["type"]]), d=d,
                 dw=V[:, 8:8 + I * O].unflatten(1, (I, O)), db=V[:, at:at + O] if case["bias"] else None)


def _pairs(case):
    """Pairs of a head's turned part for each axis: the first axis (time) takes what the others leave."""
    total = (case["dim"] - case["rest"]) // 2
    each = total // case["axes"]
    return [total - each * (case["axes"] - 1)] + [each] * (case["axes"] - 1)


def _frequencies(case):
    return [10000.0 ** (-i / n) for n in _pairs(case) for i in range(n)]


def _prepare_turn(case, gen, state):
    K, N, T, H, D, A = case["K"], case["batch"], case["tokens"], case["heads"], case["dim"], case["axes"]
    x = _normal(gen, K, N, T, H, D).to(TYPES[case["type"]])
    if case["own_positions"]:
        # sequences of different lengths: every one starts somewhere, far out along the first axis
        start = torch.randint(0, 200000, (1, K, N, 1), generator=gen, device="cuda")
        step = torch.randint(0, 2048, (A, K, N, T), generator=gen, device="cuda")
        positions = step
        positions[0] = (start + torch.arange(T, device="cuda"))[0]
    else:
        side = max(1, round((T / 16) ** 0.5)) if T >= 256 else max(1, round(T ** 0.5))
        t = torch.arange(T, device="cuda")
        places = [t // (side * side), t // side % side, t % side]      # frame, row, column
        positions = torch.stack(places[3 - A:])
    state.update(x=x, positions=positions.to(torch.int32).contiguous(), d=64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 31)
    state = dict(case=case, seed=seed + 5, call=7)
    {"norm": _prepare_norm, "keep": _prepare_keep, "grad": _prepare_grad, "turn": _prepare_turn}[case["op"]](case, gen, state)
    if own:
        # what a trainer keeps: its context, the layer's rotary plan, the activation in its 8 bits
        from paper_2308_09187_amd import qgx
        state["ctx"] = qgx.Context(state["d"], case["K"], 4096, seed=state["seed"])
        if case["op"] == "grad":
            state["kept"] = qgx.Checkpoint(state["codes"], state["powers"], case["cols"])
        if case["op"] == "turn":
            state["rotary"] = qgx.Rotary(_pairs(case), _frequencies(case), neighbours=case["neighbours"])
    return state


# -- the plain forms ----------------------------------------------------------------------------------------------------


def _philox(c0, c1, c2, c3, seed):
    """Four words of Philox4x32-10 (Salmon, Moraes, Dror, Shaw, 2011) for each counter, as whole numbers of 64 bits."""
    k0, k1, mask = seed & 0xFFFFFFFF, seed >> 32, 0xFFFFFFFF

    def product(m, x):                                     # high and low word of m x, by halves of x
        low, high = m * (x & 0xFFFF), m * (x >> 16)
        return (high + (low >> 16)) >> 16, (low + ((high & 0xFFFF) << 16)) & mask

    for r in range(10):
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ ((k0 + r * 0x9E3779B9) & mask), l1, h0 ^ c3 ^ ((k1 + r * 0xBB67AE85) & mask), l0
    return c0, c1, c2, c3


def _draws(rows, cols, seed, call):
    """16 bits for every element [rows, cols]: eight to a Philox block, counter (column / 8, 2, row, call)."""
    g = torch.arange((cols + 7) // 8, device="cuda", dtype=torch.int64).view(1, -1).expand(rows, -1)
    r = torch.arange(rows, device="cuda", dtype=torch.int64).view(-1, 1).expand_as(g)
    words = torch.stack(_philox(g, torch.full_like(g, 2), r, torch.full_like(g, call), seed), -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).flatten(-3)[:, :cols]


def _keep(x, call, seed):
    """Codes [.., up to whole blocks] and biased powers [.., blocks], both bytes, of x's rows.  A block's power of two is the smallest
    with all magnitudes at most 127 of it; a code is 128 + the element over it, rounded to nearest even, or, with a call's
    draws, away from zero where the draw is below the remainder."""
    lead, cols = x.shape[:-1], x.shape[-1]
    top = 136 if x.dtype == torch.float16 else 248         # (no value beyond the type's range)
    x = x.float().reshape(-1, cols)
    pad = -cols % BLOCK
    v = torch.nn.functional.pad(x, (0, pad)).unflatten(1, (-1, BLOCK))
    bits = v.abs().amax(2).view(torch.int32)
    power = (bits >> 23) - 6 + ((bits & 0x7FFFFF) > 0x7E0000)
    power = torch.where(bits == 0, torch.zeros_like(power), power.clamp(1, top))
    u = v * torch.where(bits == 0, torch.zeros_like(power), (254 - power) << 23).view(torch.float32).unsqueeze(2)
    if call is None:
        code = torch.round(u)
    else:
        m = u.abs()
        down = torch.floor(m)
        draw = torch.nn.functional.pad(_draws(x.shape[0], cols, seed, call), (0, pad)).view_as(v)
        code = torch.sign(u) * (down + (draw.float() < (m - down) * 65536.0))
    code = code.clamp(-127, 127)
    return (code + 128).to(torch.uint8).flatten(1).view(*lead, cols + pad), power.to(torch.uint8).view(*lead, -1)


def _values(codes, powers, cols):
    """What kept activations stand for, binary32."""
    scale = (powers.to(torch.int32) << 23).view(torch.float32)
    return ((codes.float() - 128.0).unflatten(-1, (-1, BLOCK)) * scale.unsqueeze(-1)).flatten(-2)[..., :cols]


def _plain_norm(s, x):
    c = s["case"]
    K, N, P, C, G = c["K"], c["batch"], c["places"], c["channels"], c["groups"]
    f = x.float().view(K, N, P, G, C // G)
    mean = f.mean((2, 4))
    f = f - mean.view(K, N, 1, G, 1)
    rstd = 1.0 / torch.sqrt((f * f).mean((2, 4)) + s["eps"])
    z = (f * rstd.view(K, N, 1, G, 1)).view(K, N, P, C) * s["w"] + s["b"]
    if c["act"] == "silu":
        z = z / (1.0 + torch.exp(-z))
    elif c["act"] == "leaky":
        z = torch.where(z > 0, z, s["slope"] * z)
    return z.to(x.dtype), mean, rstd


def _plain_norm_back(s, x, mean, rstd):
    c = s["case"]
    K, N, P, C, G = c["K"], c["batch"], c["places"], c["channels"], c["groups"]
    group = (K, N, 1, G, 1)
    h = ((x.float().view(K, N, P, G, C // G) - mean.view(group)) * rstd.view(group)).view(K, N, P, C)
    dz = s["dy"].float()
    if c["act"] != "none":
        z = h * s["w"] + s["b"]
        if c["act"] == "silu":
            sig = 1.0 / (1.0 + torch.exp(-z))
            dz = dz * (sig * (1.0 + z * (1.0 - sig)))
        else:
            dz = torch.where(z > 0, dz, s["slope"] * dz)
    s["dw"].copy_((dz * h).sum((1, 2)))
    s["db"].copy_(dz.sum((1, 2)))
    g = (dz * s["w"]).view(K, N, P, G, C // G)
    h = h.view_as(g)
    dx = rstd.view(group) * (g - g.mean((2, 4), keepdim=True) - h * (g * h).mean((2, 4), keepdim=True))
    return dx.view(K, N, P, C).to(s["dy"].dtype)


def _plain_turn(s):
    c = s["case"]
    D, R = c["dim"], c["dim"] - c["rest"]
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_pairs(c), device="cuda"))
    f = torch.tensor(_frequencies(c), device="cuda", dtype=torch.float64)
    angle = torch.movedim(s["positions"].double()[axis], 0, -1) * f              # [.., tokens, pairs], in 64 bits
    cos, sin = torch.cos(angle).float().unsqueeze(-2), torch.sin(angle).float().unsqueeze(-2)
    if c["back"]:
        sin = -sin
    x = s["x"].float()
    if c["neighbours"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        out = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        out = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([out, x[..., R:D]], -1).to(s["x"].dtype)


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c, s["ctx"])
    if c["op"] == "norm":
        if c["mode"] == "forward":
            y, mean, rstd = _plain_norm(s, s["x"])
            return {"y": y, "mean": mean, "rstd": rstd}
        if c["mode"] == "backward":
            return {"dx": _plain_norm_back(s, s["x"], s["mean"], s["rstd"]), "dw": s["dw"], "db": s["db"]}
        y, mean, rstd = _plain_norm(s, s["x"])
        kept = _values(*_keep(s["x"], s["call"], s["seed"]), c["channels"])
        return {"y": y, "mean": mean, "rstd": rstd, "dx": _plain_norm_back(s, kept, mean, rstd), "dw": s["dw"], "db": s["db"]}
    if c["op"] == "keep":
        codes, powers = _keep(s["x"], s["call"] if c["unbiased"] else None, s["seed"])
        return {"x": _values(codes, powers, c["cols"]).to(s["x"].dtype)}
    if c["op"] == "grad":
        x, dy = _values(s["codes"], s["powers"], c["cols"]), s["dy"].float()
        s["dw"].copy_(torch.bmm(x.transpose(1, 2), dy))
        if s["db"] is not None:
            s["db"].copy_(dy.sum(1))
        return {"dw": s["dw"], "db": s["db"]}
    return {"x": _plain_turn(s)}


def _own(s, c, ctx):
    if c["op"] == "norm":
        act = dict(activation=c["act"], slope=s["slope"])
        if c["mode"] == "backward":
            dx = ctx.group_norm_backward(s["dy"], s["x"], c["groups"], s["w"], s["b"], s["mean"], s["rstd"], dw=s["dw"], db=s["db"], **act)
            return {"dx": dx, "dw": s["dw"], "db": s["db"]}
        if c["mode"] == "forward":
            y, mean, rstd = ctx.group_norm(s["x"], c["groups"], s["w"], s["b"], s["eps"], **act)
            return {"y": y, "mean": mean, "rstd": rstd}
        kept = ctx.new_checkpoint(s["x"].shape)
        y, mean, rstd = ctx.group_norm(s["x"], c["groups"], s["w"], s["b"], s["eps"], keep=kept, call_id=s["call"], **act)
        dx = ctx.group_norm_backward(s["dy"], kept, c["groups"], s["w"], s["b"], mean, rstd, dw=s["dw"], db=s["db"], **act)
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dw": s["dw"], "db": s["db"]}
    if c["op"] == "keep":
        kept = ctx.checkpoint(s["x"], call_id=s["call"] if c["unbiased"] else None)
        return {"x": ctx.restore(kept, s["x"].dtype)}
    if c["op"] == "grad":
        ctx.weight_gradient(s["kept"], s["dy"], s["dw"], db=s["db"])
        return {"dw": s["dw"], "db": s["db"]}
    return {"x": ctx.rotary(s["x"], s["rotary"], s["positions"], back=c["back"])}


# -- what a pass cannot do without --------------------------------------------------------------------------------------


def _kept_bytes(rows, cols):
    blocks = (cols + BLOCK - 1) // BLOCK
    return rows * (cols + blocks)


def work(case):
    K = case["K"]
    if case["op"] == "norm":
        rows, C = K * case["batch"] * case["places"], case["channels"]
        n, size, stats = rows * C, SIZE[case["type"]], 8 * K * case["batch"] * case["groups"]
        forward = {"bytes": 2 * n * size + stats + 8 * C, "flops": 10 * n}
        if case["mode"] == "forward":
            return forward
        if case["mode"] == "backward":
            return {"bytes": 3 * n * size + stats + 8 * C * (1 + K), "flops": 24 * n}
        # the kept input is written by one pass and read by the other
        return {"bytes": forward["bytes"] + 2 * _kept_bytes(rows, C) + 2 * n * size + stats + 8 * C * (1 + K), "flops": 40 * n}
    if case["op"] == "keep":
        n, size = K * case["rows"] * case["cols"], SIZE[case["type"]]
        return {"bytes": 2 * n * size + 2 * _kept_bytes(K * case["rows"], case["cols"]), "flops": 6 * n}
    if case["op"] == "grad":
        rows, I, O = case["rows"], case["cols"], case["out"]
        return {"bytes": _kept_bytes(K * rows, I) + K * rows * O * SIZE[case["type"]] + 4 * K * I * O, "flops": 2 * K * rows * I * O}
    tokens = case["batch"] * K * case["tokens"]
    n = tokens * case["heads"] * case["dim"]
    own_positions = tokens if case["own_positions"] else case["tokens"]
    return {"bytes": 2 * n * SIZE[case["type"]] + 4 * case["axes"] * own_positions, "flops": 3 * n}


# -- the definitions in 64 bits -----------------------------------------------------------------------------------------


def _exact_draws(rows, cols, seed, call):
    """The draws [rows, up to eights of cols] in whole numbers of numpy's 64 bits."""
    groups = (cols + 7) // 8
    m32 = np.uint64(0xFFFFFFFF)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.full(rows * groups, 2, np.uint64),
         np.repeat(np.arange(rows, dtype=np.uint64), groups), np.full(rows * groups, call, np.uint64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & m32]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack([w.astype(np.uint32) for w in c], 1).view(np.uint16).reshape(rows, groups * 8)


def _powers_of_two(e):
    """2^e, exactly (a device's own power function may be off by its last bit)."""
    return torch.tensor([2.0 ** i for i in range(-127, 128)], dtype=torch.float64, device=e.device)[e + 127]


def _exact_keep(x, call, seed):
    """The values that x's rows are kept as: every block a whole multiple, up to 127, of its power of two."""
    cols = x.shape[-1]
    limit = 9 if x.dtype == torch.float16 else 121
    v = x.double().reshape(-1, cols)
    blocks = torch.split(v, BLOCK, dim=1)
    e = torch.stack([torch.ceil(torch.log2(p.abs().amax(1) / 127.0)) for p in blocks], 1).clamp(-126, limit)
    step = _powers_of_two(e.long().repeat_interleave(BLOCK, 1)[:, :cols])
    u = v / step
    if call is None:
        u = torch.round(u)
    else:
        r = torch.from_numpy(_exact_draws(v.shape[0], cols, seed, call)[:, :cols].astype(np.int32)).to(x.device)
        up = u.abs() - u.abs().floor() > r / 65536.0
        u = torch.where(u < 0, -1.0, 1.0) * (u.abs().floor() + up)
    return (u.clamp(-127, 127) * step).view(x.shape)


def _exact_norm(s, c):
    K, N, P, C, G = c["K"], c["batch"], c["places"], c["channels"], c["groups"]
    w, b = s["w"].double(), s["b"].double()
    out = {}

    def unit(z):
        if c["act"] == "silu":
            return z * torch.sigmoid(z), torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        if c["act"] == "leaky":
            return torch.maximum(z, s["slope"] * z), torch.where(z > 0, 1.0, s["slope"]).to(z.dtype)
        return z, torch.ones_like(z)

    if c["mode"] == "backward":
        mean, rstd = s["mean"].double(), s["rstd"].double()
    else:
        mean, rstd = torch.empty(2, K, N, G, dtype=torch.float64, device="cuda").unbind(0)
        out["y"] = torch.empty(K, N, P, C, dtype=torch.float64, device="cuda")
        for k in range(K):
            x = s["x"][k].double().view(N, P, G, C // G)
            var, mean[k] = torch.var_mean(x, dim=(1, 3), unbiased=False)
            rstd[k] = torch.rsqrt(var + s["eps"])
            h = (x - mean[k][:, None, :, None]) * rstd[k][:, None, :, None]
            out["y"][k] = unit(torch.addcmul(b, h.reshape(N, P, C), w))[0]
        out.update(mean=mean, rstd=rstd)
    if c["mode"] == "forward":
        return out
    out.update(dx=torch.empty(K, N, P, C, dtype=torch.float64, device="cuda"),
               dw=torch.empty(K, C, dtype=torch.float64, device="cuda"), db=torch.empty(K, C, dtype=torch.float64, device="cuda"))
    kept = _exact_keep(s["x"], s["call"], s["seed"]) if c["mode"] == "step" else s["x"]
    if c["mode"] == "step":
        # the activation's derivative is that of the binary32 statistics' place, as the backward pass is given them
        mean, rstd = mean.float().double(), rstd.float().double()
    for k in range(K):
        h = (kept[k].double().view(N, P, G, C // G) - mean[k][:, None, :, None]) * rstd[k][:, None, :, None]
        dz = s["dy"][k].double() * unit(torch.addcmul(b, h.reshape(N, P, C), w))[1]
        out["dw"][k], out["db"][k] = torch.sum(dz * h.reshape(N, P, C), (0, 1)), torch.sum(dz, (0, 1))
        g = (dz * w).view(N, P, G, C // G)
        n = P * (C // G)
        along, mid = torch.einsum("npgc,npgc->ng", g, h) / n, g.sum((1, 3)) / n
        dx = (g - mid[:, None, :, None] - h * along[:, None, :, None]) * rstd[k][:, None, :, None]
        out["dx"][k] = dx.reshape(N, P, C)
    return out


def _exact_turn(s, c):
    x = s["x"].double()
    R = c["dim"] - c["rest"]
    out = x.clone()
    p = 0
    for axis, n in enumerate(_pairs(c)):
        for i in range(n):
            # one pair at a time, as a complex number times exp(i angle)
            angle = s["positions"][axis].double() * 10000.0 ** (-i / n) * (-1.0 if c["back"] else 1.0)
            at = (2 * p, 2 * p + 1) if c["neighbours"] else (p, p + R // 2)
            turned = torch.complex(x[..., at[0]], x[..., at[1]]) * torch.polar(torch.ones_like(angle), angle).unsqueeze(-1)
            out[..., at[0]], out[..., at[1]] = turned.real, turned.imag
            p += 1
    return {"x": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s, case)
    if case["op"] == "keep":
        return {"x": _exact_keep(s["x"], s["call"] if case["unbiased"] else None, s["seed"])}
    if case["op"] == "turn":
        return _exact_turn(s, case)
    K, I = case["K"], case["cols"]
    dw = torch.empty(K, I, case["out"], dtype=torch.float64, device="cuda")
    for k in range(K):
        step = _powers_of_two(s["powers"][k].long() - 127).repeat_interleave(BLOCK, 1)
        x = ((s["codes"][k].double() - 128.0) * step)[:, :I]
        dw[k] = torch.matmul(x.t(), s["dy"][k].double())
    return {"dw": dw, "db": s["dy"].double().sum(1) if case["bias"] else None}
