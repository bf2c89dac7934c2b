"""The parts of a gated, rotary block around graph self-attention, as cases that can be timed.

  rotary  rotary positions on Q and K: a rotation of feature pairs by an angle that grows with the node's position,
          forward, or forward and backward (a rotation the other way)
  norm    y = residual_scale * x + gate * norm(branch) and h = norm(y): the norm after a block, its gate, the residual
          sum and the norm before the next block in one pass; forward, or forward and backward
  ffn     Y = (act(X Wg) * (X Wu)) Wd: the gated feed-forward block, forward, or forward and backward

`listed()` spans the sizes of paper_1911_04070_amd/workloads.py and bench.py (8 heads of 64, d = 512, trees over 512,
2048 and 8192 tokens, 32 sentences of very different lengths) and wider layers; `draw()` gives other sizes of the same
ranges.  States, queries, keys and gradients are N(0, 1), parameters as a fresh block has them.

`run` computes the plain form with elementary torch operations in fp32 (angles in fp64), rounded once at the end; with
`own` set it makes the framework's calls.
"""
import math

import torch

own = False

HEAD = 64
BASE = 10000.0
EPS = 1e-5


def listed():
    return [
        # one new token for each of 32 sequences, far into a long context: a decoding step, nothing but latency
        dict(name="rotary_token", op="rotary", B=32, H=8, N=1, rot=64, interleaved=False, factor=4.0, context=8192,
             pos="each", far=32768, dtype="bf16", packed=False, backward=False),
        # the nodes of 2 trees over 2048 tokens in fp32, half of the head rotated, pairs side by side
        dict(name="rotary_f32", op="rotary", B=2, H=8, N=4095, rot=32, interleaved=True, factor=1.0, context=0,
             pos="nodes", far=2048, dtype="f32", packed=False, backward=False),
        # a training step on the language-model shape: Q and K side by side in the rows a projection writes
        dict(name="rotary_lm", op="rotary", B=4, H=8, N=16383, rot=64, interleaved=False, factor=1.0, context=0,
             pos="nodes", far=8192, dtype="bf16", packed=True, backward=True),
        # between two blocks of a decoding step for 8 sequences
        dict(name="norm_token", op="norm", rows=8, d=512, post="rms", pre="rms", gate_rows=8, dtype="bf16", backward=False),
        # the rows of 32 sentences packed into one graph, a gate for every row
        dict(name="norm_sentences", op="norm", rows=15003, d=512, post="layer", pre="layer", gate_rows=1, dtype="bf16", backward=False),
        # a training step between two blocks on the language-model shape, a gate for each of the 4 sequences
        dict(name="norm_lm", op="norm", rows=65532, d=512, post="rms", pre="rms", gate_rows=16383, dtype="bf16", backward=True),
        # the same in fp32 on a wider block, a learned gate shared by all rows
        dict(name="norm_wide_f32", op="norm", rows=4095, d=2048, post="layer", pre="layer", gate_rows=4095, dtype="f32", backward=True),
        # a decoding step: one row through the block, bound by reading the weights
        dict(name="ffn_token", op="ffn", rows=1, d=512, f=1368, act="silu", backward=False),
        # the rows of 32 sentences packed into one graph, inference
        dict(name="ffn_sentences", op="ffn", rows=15003, d=512, f=1368, act="silu", backward=False),
        # a training step on one tree over 512 tokens: few rows
        dict(name="ffn_small", op="ffn", rows=1023, d=512, f=1368, act="gelu", backward=True),
        # a training step on the language-model shape
        dict(name="ffn_lm", op="ffn", rows=65532, d=512, f=2048, act="silu", backward=True),
        # a wide block on a batch of 8 sentences of up to 1024 tokens
        dict(name="ffn_wide", op="ffn", rows=9001, d=2048, f=5464, act="silu", backward=True),
    ]


def draw(rng):
    def size(lo, hi):        # whole number, its logarithm spread evenly, odd ones among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "norm", "ffn"])
    if op == "rotary":
        dtype = rng.choice(["f32", "bf16", "bf16"])
        H = rng.choice([1, 2, 3, 4, 6, 8, 8, 12, 16])
        N = size(1, 16383)
        B = size(1, max(1, min(32, (1 << 19) // (H * N))))
        pos = rng.choice(["nodes", "each"])
        return dict(op=op, B=B, H=H, N=N, rot=rng.choice([16, 24, 32, 48, 64, 64]), interleaved=rng.random() < 0.5,
                    factor=rng.choice([1.0, 1.0, 2.0, 4.0, 8.0]), context=rng.choice([0, 2048, 8192]), pos=pos,
                    far=size(N + 1, 1 << 20) if pos == "each" else N, dtype=dtype, packed=rng.random() < 0.5,
                    backward=rng.random() < 0.5)
    if op == "norm":
        dtype = rng.choice(["f32", "bf16", "bf16"])
        d = 8 * size(8, 512)
        rows = size(1, max(2, min(65532, (1 << 25) // d // (2 if dtype == "f32" else 1))))
        return dict(op=op, rows=rows, d=d, post=rng.choice(["layer", "rms", "rms", "none"]), pre=rng.choice(["layer", "rms"]),
                    gate_rows=rng.choice([0, 1, size(1, rows), rows]), dtype=dtype, backward=rng.random() < 0.6)
    d = 64 * size(1, 32)
    f = 8 * size(16, min(1024, 3 * d // 8))
    rows = size(1, max(2, min(65532, (1 << 36) // (d * f))))
    return dict(op=op, rows=rows, d=d, f=f, act=rng.choice(["silu", "gelu", "relu"]), backward=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype, std=1.0):
    x = torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32)
    return (x if std == 1.0 else x.mul_(std)).to(dtype)


def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _node_positions(N):
    """Centre of every node's tokens, nodes level by level: tokens 0, 1, 2, ..., spans of two 0.5, 2.5, ... (the first N)."""
    rows, width, count = [], 1, (N + 1) // 2
    while sum(len(r) for r in rows) < N:
        rows.append(torch.arange(max(count, 1), dtype=torch.float64) * width + (width - 1) / 2)
        width, count = 2 * width, count // 2
    return torch.cat(rows)[:N].to(torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(case)
    s = dict(case=case)
    if case["op"] == "rotary":
        B, H, N = case["B"], case["H"], case["N"]
        wanted = ("Q", "K", "dQ", "dK") if case["backward"] else ("Q", "K")
        if case["packed"]:   # a row holds the queries, keys, values and outputs of all heads, as a projection writes them
            for a, b in (("Q", "K"), ("dQ", "dK"))[: len(wanted) // 2]:
                x = _normal(gen, (B, N, 4, H, HEAD), dt)
                s[a], s[b] = (x[:, :, i].permute(0, 2, 1, 3) for i in range(2))
        else:
            for name in wanted:
                s[name] = _normal(gen, (B, H, N, HEAD), dt)
        if case["pos"] == "nodes":
            s["pos"] = _node_positions(N).cuda()
        else:
            start = torch.randint(0, case["far"] - N + 1, (B, 1), device="cuda", generator=gen)
            s["pos"] = (start + torch.arange(N, device="cuda")).to(torch.float32)
    elif case["op"] == "norm":
        rows, d, g = case["rows"], case["d"], case["gate_rows"]
        for name in ("x", "branch") + (("dy", "dh") if case["backward"] else ()):
            s[name] = _normal(gen, (rows, d), dt)
        s["gate"] = _normal(gen, (-(-rows // g), d), dt) if g else None
        for which in ("post", "pre"):
            has = case[which] != "none"
            s[which + "_gain"] = 1.0 + _normal(gen, (d,), torch.float32, 0.1) if has else None
            s[which + "_bias"] = _normal(gen, (d,), torch.float32, 0.1) if case[which] == "layer" else None
        s["residual_scale"] = 0.5 ** 0.5
    else:
        rows, d, f = case["rows"], case["d"], case["f"]
        s["X"] = _normal(gen, (rows, d), dt)
        s["Wg"], s["Wu"] = (_normal(gen, (d, f), dt, d ** -0.5) for _ in range(2))
        s["Wd"] = _normal(gen, (f, d), dt, f ** -0.5)
        if case["backward"]:
            s["dY"] = _normal(gen, (rows, d), dt)
    return s


def run(state):
    return {"rotary": _run_rotary, "norm": _run_norm, "ffn": _run_ffn}[state["case"]["op"]](state)


# ---- rotary positions -----------------------------------------------------------------------------------
def _run_rotary(s):
    c = s["case"]
    if own:
        from paper_1911_04070_amd import binding as bpt
        how = dict(rot=c["rot"], interleaved=c["interleaved"], base=BASE, factor=c["factor"], context=c["context"])
        out = bpt.bpt_rotary(s["Q"], s["K"], s["pos"], **how)
        if c["backward"]:
            out = out + bpt.bpt_rotary(s["dQ"], s["dK"], s["pos"], inverse=True, **how)
        return out
    # theta_i = base^(-2i / rot); pairs that turn fewer than `low` times over the original context are slowed down by
    # the factor, pairs that turn more than `high` times are left alone, between the two linearly
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    theta = torch.exp(i * (-2.0 / c["rot"] * math.log(BASE)))
    keep = (theta * (c["context"] / (2 * math.pi)) - 1.0) / (32.0 - 1.0)
    keep = keep.clamp(0.0, 1.0) if c["context"] else torch.zeros_like(theta)
    theta = theta * (keep + (1.0 - keep) / c["factor"])
    pos = s["pos"].double()
    angle = (pos if pos.dim() == 2 else pos[None])[:, None, :, None] * theta
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turn(x, sin):
        y = x.float().clone(memory_format=torch.contiguous_format)
        h = c["rot"] // 2
        at = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else (slice(0, h), slice(h, c["rot"]))
        a, b = x[..., at[0]].float(), x[..., at[1]].float()
        y[..., at[0]] = a * cos - b * sin
        y[..., at[1]] = b * cos + a * sin
        return y.to(x.dtype)

    out = (turn(s["Q"], sin), turn(s["K"], sin))
    return out + (turn(s["dQ"], -sin), turn(s["dK"], -sin)) if c["backward"] else out


def _exact_rotary(c, s):
    freq = torch.tensor([BASE ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)], dtype=torch.float64)
    for i in range(len(freq)):
        w = float(freq[i])
        turns = c["context"] * w / (2 * math.pi)
        share = min(1.0, max(0.0, (turns - 1.0) / 31.0)) if c["context"] else 0.0   # of the pair that is left as it is
        freq[i] = share * w + (1.0 - share) * w / c["factor"]
    angle = torch.as_tensor(s["pos"], dtype=torch.float64).reshape(-1, 1, c["N"], 1) * freq.cuda()

    def turn(x, sign):
        x = x.double()
        head, tail = x[..., : c["rot"]], x[..., c["rot"]:]
        pairs = head.unflatten(-1, (-1, 2)) if c["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), sign * angle))
        z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, tail], -1)

    out = (turn(s["Q"], 1.0), turn(s["K"], 1.0))
    return out + (turn(s["dQ"], -1.0), turn(s["dK"], -1.0)) if c["backward"] else out


# ---- norms, gate and residual sum -----------------------------------------------------------------------
def _run_norm(s):
    c = s["case"]
    if own:
        from paper_1911_04070_amd import binding as bpt
        what = (s["x"], s["branch"], s["gate"])
        how = dict(post=c["post"], pre=c["pre"], post_gain=s["post_gain"], post_bias=s["post_bias"], pre_gain=s["pre_gain"],
                   pre_bias=s["pre_bias"], gate_rows=c["gate_rows"], residual_scale=s["residual_scale"], eps=EPS)
        if not c["backward"]:
            return bpt.bpt_residual_norm_fwd(*what, **how)
        y, h, stats = bpt.bpt_residual_norm_fwd(*what, want_stats=True, **how)
        return {"y": y, "h": h, **bpt.bpt_residual_norm_bwd(*what, stats, s["dy"], s["dh"], **how)}
    dt, rows, d = s["x"].dtype, c["rows"], c["d"]

    def normed(v, kind):
        if kind == "none":
            return v, None
        if kind == "layer":
            v = v - v.mean(-1, keepdim=True)
        r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        return v * r, r

    def spread(vhat, kind, which):
        out = vhat if kind == "none" else vhat * s[which + "_gain"]
        return out if s[which + "_bias"] is None else out + s[which + "_bias"]

    gate = None
    if c["gate_rows"]:
        gate = s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:rows]
    bhat, rb = normed(s["branch"].float(), c["post"])
    b = spread(bhat, c["post"], "post")
    y = s["residual_scale"] * s["x"].float() + (b if gate is None else gate * b)
    yhat, ry = normed(y, c["pre"])
    h = spread(yhat, c["pre"], "pre")
    if not c["backward"]:
        return y.to(dt), h.to(dt)

    def back(g, vhat, r, kind, which):      # gradient of spread(normed(v)) with respect to v, gain and bias
        if kind == "none":
            return g, {}
        grads = {"d_%s_gain" % which: (g * vhat).double().sum(0).float()}
        if s[which + "_bias"] is not None:
            grads["d_%s_bias" % which] = g.double().sum(0).float()
        g = g * s[which + "_gain"]
        dv = g - vhat * (g * vhat).mean(-1, keepdim=True)
        if kind == "layer":
            dv = dv - g.mean(-1, keepdim=True)
        return dv * r, grads

    dv, grads = back(s["dh"].float(), yhat, ry, c["pre"], "pre")
    dy = s["dy"].float() + dv
    out = {"y": y.to(dt), "h": h.to(dt), "dx": (s["residual_scale"] * dy).to(dt)}
    if gate is not None:
        groups = s["gate"].shape[0]
        pad = torch.zeros(groups * c["gate_rows"], d, dtype=torch.float64, device="cuda")
        pad[:rows] = (dy * b).double()
        out["d_gate"] = pad.view(groups, c["gate_rows"], d).sum(1).to(dt)
    db, more = back(dy if gate is None else dy * gate, bhat, rb, c["post"], "post")
    out["d_branch"] = db.to(dt)
    return {**out, **grads, **more}


def _exact_norm(c, s):
    leaf = {k: v.double().requires_grad_(c["backward"]) for k, v in s.items() if isinstance(v, torch.Tensor)}

    def norm(v, which):
        if c[which] == "none":
            return v
        centre = v.mean(1, keepdim=True) if c[which] == "layer" else torch.zeros((), dtype=torch.float64, device="cuda")
        v = (v - centre) / torch.sqrt(((v - centre) ** 2).sum(1, keepdim=True) / c["d"] + EPS) * leaf[which + "_gain"]
        return v + leaf[which + "_bias"] if which + "_bias" in leaf else v

    b = norm(leaf["branch"], "post")
    if "gate" in leaf:
        b = b * leaf["gate"][torch.arange(c["rows"], device="cuda") // c["gate_rows"]]
    y = leaf["x"] * s["residual_scale"] + b
    h = norm(y, "pre")
    if not c["backward"]:
        return y, h
    names = [k for k in ("x", "branch", "gate", "post_gain", "post_bias", "pre_gain", "pre_bias") if k in leaf]
    grads = torch.autograd.grad((y * leaf["dy"].detach()).sum() + (h * leaf["dh"].detach()).sum(), [leaf[k] for k in names])
    return {"y": y.detach(), "h": h.detach(), **{("d" if k == "x" else "d_") + k: g for k, g in zip(names, grads)}}


# ---- gated feed-forward block ---------------------------------------------------------------------------
def _run_ffn(s):
    c = s["case"]
    if own:
        from paper_1911_04070_amd import binding as bpt
        Y = bpt.bpt_gated_ffn_fwd(s["X"], s["Wg"], s["Wu"], s["Wd"], activation=c["act"])
        if not c["backward"]:
            return Y
        return (Y,) + bpt.bpt_gated_ffn_bwd(s["X"], s["Wg"], s["Wu"], s["Wd"], s["dY"], activation=c["act"], bf16_grads=True)
    dt = s["X"].dtype
    X, Wg, Wu, Wd = (s[k].float() for k in ("X", "Wg", "Wu", "Wd"))
    g, u = X @ Wg, X @ Wu
    if c["act"] == "silu":
        share = 1.0 / (1.0 + torch.exp(-g))
    elif c["act"] == "gelu":
        share = 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5))
    else:
        share = (g > 0).float()
    a = g * share
    F = a * u
    Y = (F @ Wd).to(dt)
    if not c["backward"]:
        return Y
    if c["act"] == "silu":
        slope = share * (1.0 + g * (1.0 - share))
    elif c["act"] == "gelu":
        slope = share + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    else:
        slope = share
    dY = s["dY"].float()
    dF = dY @ Wd.t()
    dg, du = dF * u * slope, dF * a
    return (Y, (dg @ Wg.t() + du @ Wu.t()).to(dt), (X.t() @ dg).to(dt), (X.t() @ du).to(dt), (F.t() @ dY).to(dt))


def _exact_ffn(c, s):
    leaf = [s[k].double().requires_grad_(c["backward"]) for k in ("X", "Wg", "Wu", "Wd")]
    g, u = leaf[0].mm(leaf[1]), leaf[0].mm(leaf[2])
    if c["act"] == "silu":
        a = g * torch.sigmoid(g)
    elif c["act"] == "gelu":
        a = g * torch.special.ndtr(g)
    else:
        a = torch.where(g > 0, g, torch.zeros_like(g))
    Y = (a * u).mm(leaf[3])
    return (Y.detach(),) + torch.autograd.grad(Y, leaf, s["dY"].double()) if c["backward"] else Y


def exact(case, seed):
    return {"rotary": _exact_rotary, "norm": _exact_norm, "ffn": _exact_ffn}[case["op"]](case, prepare(case, seed))


# ---- what a pass cannot do without ----------------------------------------------------------------------
def work(case):
    width = 4 if case.get("dtype") == "f32" else 2
    ways = 2 if case["backward"] else 1
    if case["op"] == "rotary":
        rows = case["B"] * case["H"] * case["N"]
        pos = 4 * case["N"] * (case["B"] if case["pos"] == "each" else 1)
        return {"bytes": ways * (2 * 2 * rows * HEAD * width + pos), "flops": ways * 2 * rows * 3 * case["rot"]}
    if case["op"] == "norm":
        rows, d, g = case["rows"], case["d"], case["gate_rows"]
        gate = -(-rows // g) * d * width if g else 0
        # forward: x, branch -> y, h; backward: x, branch, dy, dh -> dx, d_branch; the gate and its gradient
        size = rows * d * width * (10 if case["backward"] else 4) + gate * (3 if case["backward"] else 1)
        return {"bytes": size, "flops": rows * d * (44 if case["backward"] else 14)}
    rows, d, f = case["rows"], case["d"], case["f"]
    size = 2 * (2 * rows * d + 3 * d * f)
    if case["backward"]:      # the step reads X, dY and the weights and writes Y, dX and the weights' gradients
        size = 2 * (4 * rows * d + 6 * d * f)
    return {"bytes": size, "flops": 6 * rows * d * f * (3 if case["backward"] else 1)}
