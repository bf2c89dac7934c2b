"""Norms before and after a sublayer with gate and residual sum, against formulas in 64 bits.

Tolerances.  u = 2^-24 is fp32's half step.  A row's mean and mean square are sums of d terms in a tree of at most 8 adds in a
thread and log2(d / 8) levels over threads (<= 17 roundings), the normalised value takes a dozen more: 64 u of the largest
entry of the result is used for y and h, four times that for the gradients of x and branch, whose formula chains two such norms
and subtracts means.  Column sums add terms p q, p a gradient (dY, dN or dh) and q a normalised row (or 1): p may be
off by the 256 u max|p| and q by the 64 u max(1, |q|) just stated -- not by a share of their own value, p being a difference
that can come out near zero -- so a term is off by |q| 256 u max|p| + |p| 64 u max(1, |q|), and adding them (a handful of rows
per thread, the rest in trees) costs 128 u of the sum of |p q|.  Results in bf16 are rounded once more: 2^-8 relative.
"""
import pytest
import torch

from paper_1911_04070_amd import binding as bpt

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
EPS = 1e-5


def make(rows, d, dtype, post, pre, gate_rows, seed, branch=True, biases=True, alpha=0.75):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    c = dict(post=post, pre=pre, gate_rows=gate_rows, residual_scale=alpha)
    t = dict(x=r(rows, d).to(dtype), branch=r(rows, d).to(dtype) if branch else None,
             gate=r(-(-rows // gate_rows), d).to(dtype) if gate_rows else None)
    for w, kind in (("post", post), ("pre", pre)):
        t[w + "_gain"] = 1 + 0.1 * r(d) if kind != "none" else None
        t[w + "_bias"] = 0.1 * r(d) if kind != "none" and biases else None
    t["dy"], t["dh"] = r(rows, d).to(dtype), r(rows, d).to(dtype) if pre != "none" else None
    return c, {k: v.cuda() if v is not None else None for k, v in t.items()}


def formulas(c, t):
    """y, h and the gradients, and for each column sum how far it may be off (before its rounding), fp64."""
    f = {k: v.double() if v is not None else None for k, v in t.items()}
    rows, d = t["x"].shape

    def norm(v, kind):
        if kind == "none":
            return v, torch.ones((), dtype=torch.float64, device=v.device)
        v = v - v.mean(1, keepdim=True) if kind == "layer" else v
        r = 1 / ((v * v).mean(1, keepdim=True) + EPS).sqrt()
        return v * r, r

    def spread(v, w):
        v = v * f[w + "_gain"] if f[w + "_gain"] is not None else v
        return v + f[w + "_bias"] if f[w + "_bias"] is not None else v

    gate = f["gate"][torch.arange(rows, device="cuda") // c["gate_rows"]] if c["gate_rows"] else 1.0
    bhat, rb = norm(f["branch"], c["post"]) if f["branch"] is not None else (None, None)
    bn = spread(bhat, "post") if bhat is not None else torch.zeros_like(f["x"])
    y = c["residual_scale"] * f["x"] + gate * bn
    yhat, ry = norm(y, c["pre"])
    out, size = {"y": y}, {}
    if c["pre"] != "none":
        out["h"] = spread(yhat, "pre")

    def column(name, p, q, add=lambda v: v.sum(0)):
        q = torch.ones_like(p) if q is None else q
        out[name] = add(p * q)
        size[name] = U * (128 * add((p * q).abs()) + 256 * float(p.abs().max()) * add(q.abs()) +
                          64 * max(1.0, float(q.abs().max())) * add(p.abs()))

    def back(g, vhat, r, w):
        if c[w] == "none":
            return g
        for name, q in (("_gain", vhat), ("_bias", None)):
            if f[w + name] is not None and rows:
                column("d_" + w + name, g, q)
        g = g * f[w + "_gain"] if f[w + "_gain"] is not None else g
        return r * (g - (g.mean(1, keepdim=True) if c[w] == "layer" else 0) - vhat * (g * vhat).mean(1, keepdim=True))

    dy = f["dy"] if f["dy"] is not None else torch.zeros_like(y)
    dy = dy + back(f["dh"] if f["dh"] is not None else torch.zeros_like(y), yhat, ry, "pre")
    out["dx"] = c["residual_scale"] * dy
    if f["branch"] is not None:
        if c["gate_rows"]:
            def groups(v):
                padded = torch.zeros((t["gate"].shape[0] * c["gate_rows"], d), dtype=torch.float64, device="cuda")
                padded[:rows] = v
                return padded.view(-1, c["gate_rows"], d).sum(1)

            column("d_gate", dy, bn, groups)
        out["d_branch"] = back(dy * gate, bhat, rb, "post")
    return out, size


def check(got, want, size, dtype):
    assert set(got) == set(want), (sorted(got), sorted(want))
    for name, w in want.items():
        err = (got[name].double() - w).abs()
        if name in size:
            bound = size[name]
        else:
            bound = (64 if name in ("y", "h") else 256) * U * max(1.0, float(w.abs().max()))
        if got[name].dtype == torch.bfloat16:
            bound = bound + HALF_STEP[torch.bfloat16] * w.abs()
        assert bool((err <= bound).all()), (name, float((err - bound).max()), float(err.max()))


def call(c, t):
    params = {k: t[k] for k in ("post_gain", "post_bias", "pre_gain", "pre_bias")}
    y, h, stats = bpt.bpt_residual_norm_fwd(t["x"], t["branch"], t["gate"], want_stats=True, **params, **c)
    got = {"y": y, **({"h": h} if h is not None else {})}
    if t["dy"] is not None or t["dh"] is not None:
        got.update(bpt.bpt_residual_norm_bwd(t["x"], t["branch"], t["gate"], stats, t["dy"], t["dh"], **params, **c))
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d", [(1, 8), (2, 64), (5, 120), (33, 128), (300, 136), (7, 256), (1000, 512), (63, 520), (130, 1000),
                                    (9, 2048), (2100, 264), (17, 2056), (6, 4096)])
def test_rows_and_widths(rows, d, dtype):
    for i, (post, pre, gate_rows) in enumerate((("rms", "rms", 0), ("layer", "layer", rows), ("rms", "layer", 1), ("none", "rms", 3),
                                                ("layer", "none", 7), ("none", "none", 0))):
        print("residual norm", rows, d, dtype, post, pre, gate_rows, flush=True)
        c, t = make(rows, d, dtype, post, pre, gate_rows, rows + d + i)
        check(call(c, t), *formulas(c, t), dtype)


@pytest.mark.parametrize("rows,gate_rows", [(1, 5), (9, 2), (4000, 2), (4001, 1300), (3000, 3001), (5000, 9), (700, 699)])
def test_gates_of_groups_of_rows(rows, gate_rows):
    for dtype, d in ((torch.bfloat16, 64), (torch.float32, 512), (torch.bfloat16, 600)):
        print("gates", rows, gate_rows, dtype, d, flush=True)
        c, t = make(rows, d, dtype, "rms", "layer", gate_rows, rows + gate_rows)
        check(call(c, t), *formulas(c, t), dtype)


def test_what_may_be_left_out():
    for dtype in (torch.bfloat16, torch.float32):
        c, t = make(50, 192, dtype, "none", "rms", 0, 1, branch=False)       # the norm before the first sublayer
        check(call(c, t), *formulas(c, t), dtype)
        c, t = make(50, 192, dtype, "layer", "rms", 50, 2, biases=False)
        for name in ("post_gain", "pre_gain"):
            t[name] = None
        check(call(c, t), *formulas(c, t), dtype)
        for missing in ("dy", "dh"):
            c, t = make(50, 192, dtype, "rms", "layer", 1, 3)
            t[missing] = None
            check(call(c, t), *formulas(c, t), dtype)
        c, t = make(0, 192, dtype, "rms", "layer", 0, 4)                      # no rows: zero gradients of the parameters
        got = call(c, t)
        assert got["dx"].shape == (0, 192)
        for name in ("d_post_gain", "d_post_bias", "d_pre_gain", "d_pre_bias"):
            assert bool((got[name] == 0).all())


def test_rows_without_spread_and_rows_far_from_zero():
    # zero rows, constant rows (their deviation is sqrt(eps)); a mean of 100 deviations costs that many units of the result
    c, t = make(64, 256, torch.float32, "layer", "layer", 0, 9, alpha=0.0)
    t["branch"][3] = 0
    t["branch"][5] = 2.5
    want, size = formulas(c, t)
    got = call(c, t)
    for name in ("y", "h"):
        assert float((got[name].double() - want[name]).abs().max()) <= 64 * U * (1 + 2.5 / EPS ** 0.5) * max(1.0, float(want[name].abs().max()))
    c, t = make(64, 256, torch.float32, "layer", "none", 0, 10, alpha=0.0)
    t["branch"] += 100.0
    want, size = formulas(c, t)
    y = call(c, t)["y"]
    assert float((y.double() - want["y"]).abs().max()) <= 64 * U * 100 * float(want["y"].abs().max())


def test_a_row_that_is_not_finite_stays_alone_and_strides_leave_gaps():
    c, t = make(40, 512, torch.bfloat16, "rms", "rms", 1, 11)
    want, _ = formulas(c, t)
    frame = {k: torch.full((42, 600), 9.0, dtype=torch.bfloat16, device="cuda") for k in ("x", "branch", "dy", "dh")}
    for k, v in frame.items():
        v[1:41, 8:520] = t[k]
        t[k] = v[1:41, 8:520]
    check(call(c, t), *formulas(c, t), torch.bfloat16)
    t["branch"][7, 3] = float("nan")
    t["x"][9, 0] = float("inf")
    got = call(c, t)
    rest = [i for i in range(40) if i not in (7, 9)]
    for name in ("y", "h", "dx", "d_branch", "d_gate"):
        assert bool(torch.isfinite(got[name][rest]).all())
    assert bool(torch.isnan(got["h"][7]).all())
    assert torch.equal(got["y"][rest].double(), call(c, t)["y"][rest].double())


def test_in_place_through_the_c_abi():
    c, t = make(200, 520, torch.bfloat16, "rms", "layer", 0, 12)
    want, size = formulas(c, t)
    import ctypes
    L = bpt.load_library()
    s = bpt.BptResidualNorm(200, 520, bpt.BPT_BF16, 520, 2, 1, 0, 0.75, 0.0)
    p = lambda k: t[k].data_ptr()
    x, branch = t["x"].clone(), t["branch"].clone()
    st = torch.empty((200, 4), dtype=torch.float32, device="cuda")
    stream = int(torch.cuda.current_stream().cuda_stream)
    assert L.bpt_residual_norm_fwd(ctypes.byref(s), x.data_ptr(), branch.data_ptr(), None, p("post_gain"), p("post_bias"), p("pre_gain"),
                                   p("pre_bias"), x.data_ptr(), branch.data_ptr(), st.data_ptr(), stream) == 0
    check({"y": x, "h": branch}, {k: want[k] for k in ("y", "h")}, {}, torch.bfloat16)
    # only h, no stats
    h = torch.empty_like(x)
    assert L.bpt_residual_norm_fwd(ctypes.byref(s), p("x"), p("branch"), None, p("post_gain"), p("post_bias"), p("pre_gain"), p("pre_bias"),
                                   None, h.data_ptr(), None, stream) == 0
    assert torch.equal(h, branch)
    # dx over dy, d_branch over dh
    dy, dh = t["dy"].clone(), t["dh"].clone()
    sums = [torch.empty(520, device="cuda") for _ in range(4)]
    grads = bpt.BptResidualNormGrads(None, *[v.data_ptr() for v in sums])
    need = L.bpt_residual_norm_bwd_workspace(ctypes.byref(s))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert L.bpt_residual_norm_bwd(ctypes.byref(s), p("x"), p("branch"), None, p("post_gain"), p("post_bias"), p("pre_gain"), p("pre_bias"),
                                   st.data_ptr(), dy.data_ptr(), dh.data_ptr(), dy.data_ptr(), dh.data_ptr(), ctypes.byref(grads),
                                   ws.data_ptr(), need, stream) == 0
    names = ("d_post_gain", "d_post_bias", "d_pre_gain", "d_pre_bias")
    got = {"dx": dy, "d_branch": dh, **dict(zip(names, sums))}
    check(got, {k: want[k] for k in got}, size, torch.bfloat16)


def test_gradients_against_differences():
    # directional derivatives of sum(y dy + h dh) in fp32: a step of 2^-10 leaves a second-order error near 2^-20 of curvatures
    # of order 10, and the two sums' rounding 2^-24 * sum of magnitudes / step
    c, t = make(6, 64, torch.float32, "layer", "rms", 2, 13)
    names = [k for k in ("x", "branch", "gate", "post_gain", "post_bias", "pre_gain", "pre_bias") if t[k] is not None]
    leaves = {k: t[k].clone().requires_grad_() for k in names}
    y, h = bpt.residual_norm(leaves["x"], leaves["branch"], leaves["gate"], post_gain=leaves["post_gain"], post_bias=leaves["post_bias"],
                             pre_gain=leaves["pre_gain"], pre_bias=leaves["pre_bias"], **c)
    grads = torch.autograd.grad((y * t["dy"]).sum() + (h * t["dh"]).sum(), [leaves[k] for k in names])

    def value(moved):
        w, _ = formulas(c, {**t, **moved})
        return float((w["y"] * t["dy"].double()).sum() + (w["h"] * t["dh"].double()).sum())

    for name, g in zip(names, grads):
        v = torch.randn(g.shape, generator=torch.Generator().manual_seed(3)).cuda().double()
        step = 2.0 ** -10
        slope = (value({name: t[name].double() + step * v}) - value({name: t[name].double() - step * v})) / (2 * step)
        assert abs(slope - float((g.double() * v).sum())) <= 1e-3 * max(1.0, float((g.double() * v).abs().sum())), name


def test_results_are_the_same_twice_and_in_a_replayed_graph():
    c, t = make(3001, 512, torch.bfloat16, "rms", "rms", 1000, 14)
    want = call(c, t)
    again = call(c, t)
    assert all(torch.equal(want[k], again[k]) for k in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call(c, t)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = call(c, t)
    torch.cuda.synchronize()
    for _ in range(3):
        for v in got.values():
            v.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[k], got[k]) for k in want)
        assert all(torch.equal(want[k], v) for k, v in call(c, t).items())


@pytest.mark.parametrize("rows,d,gate_rows", [(3000, 8, 0), (20011, 56, 7), (9001, 64, 100), (30000, 512, 100), (65532, 64, 2)])
def test_narrow_rows_and_many_gates(rows, d, gate_rows):
    print("residual norm", rows, d, gate_rows, flush=True)
    for dtype in (torch.bfloat16, torch.float32):
        c, t = make(rows, d, dtype, "rms", "layer", gate_rows, rows + d)
        check(call(c, t), *formulas(c, t), dtype)


def test_rows_far_into_memory():
    # rows whose elements lie more than 2^31 apart
    rows, d, stride = 1100000, 64, 2048
    c, t = make(rows, d, torch.bfloat16, "rms", "layer", 1000, 11)
    for k in ("x", "branch", "dy", "dh"):
        t[k] = torch.empty((rows, stride), dtype=torch.bfloat16, device="cuda")[:, :d].copy_(t[k])
    check(call(c, t), *formulas(c, t), torch.bfloat16)


def test_second_derivatives_are_refused():
    x = torch.randn((4, 64), device="cuda").requires_grad_()
    y, h = bpt.residual_norm(x, x)
    g, = torch.autograd.grad(h.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d", [(40, 64), (40, 512), (37, 1032), (300, 24)])
def test_rows_beside_one_that_is_not_finite_keep_their_bits(rows, d, dtype):
    # what the other rows have is compared with the call before anything was poisoned
    for post, pre in (("rms", "rms"), ("layer", "layer"), ("none", "rms")):
        c, t = make(rows, d, dtype, post, pre, 1, rows + d)
        want = call(c, t)
        for i, (name, value) in enumerate((("branch", float("nan")), ("x", float("inf")), ("dy", float("nan")), ("dh", float("-inf")),
                                           ("gate", float("inf")))):
            row = (7 * i + 3) % rows
            poisoned = dict(t, **{name: t[name].clone()})
            poisoned[name][row, d // 2 + 1] = value
            got = call(c, poisoned)
            rest = torch.arange(rows, device="cuda") != row
            for k in ("y", "h", "dx", "d_branch", "d_gate"):
                assert torch.equal(got[k][rest], want[k][rest]), (post, pre, name, k)
            assert not bool(torch.isfinite(got["dx"][row]).all()), (post, pre, name)
