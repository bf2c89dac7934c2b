"""Gated feed-forward block against formulas in 64 bits.

Tolerances.  The hidden activations F and their gradients dG, dU are rounded to bf16 once, at most 2^-8 relative each, before
the product that takes them; a result's error is therefore at most 2^-8 times the product of magnitudes (sum_k |F_k| |Wd_k| and
so on), to which the fp32 sums add less than K 2^-24 of the same, and the activation (exp, erf in fp32) and the sums under it less
than 2^-16: 1.1 * 2^-8 of the product of magnitudes is used.  Results in bf16 are rounded once more, 2^-8 relative.  Over a whole
tensor errors of random sign do not add up: its 2-norm is off by at most 2^-8 for each of the two roundings.
"""
import pytest
import torch

from paper_1911_04070_amd import binding as bpt

pytestmark = pytest.mark.gpu
H = 2.0 ** -8


def make(rows, d, f, seed, gap=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    frame = [torch.full((rows + 2, d + gap), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    X, dY = (v[1:rows + 1, :d] for v in frame)
    X.copy_(r(rows, d))
    dY.copy_(r(rows, d))
    W = [(r(d, f) * d ** -0.5).bfloat16(), (r(d, f) * d ** -0.5).bfloat16(), (r(f, d) * f ** -0.5).bfloat16()]
    return X, dY, W


def act(g, name):
    """act(g), act'(g) in fp64"""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        s = torch.special.ndtr(g)
        return g * s, s + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    return g.clamp(min=0), (g > 0).double()


def formulas(X, dY, W, name):
    """{result: (value, product of magnitudes)}"""
    X, dY, Wg, Wu, Wd = (v.double() for v in (X, dY, *W))
    g, u = X @ Wg, X @ Wu
    a, slope = act(g, name)
    F, dF = a * u, dY @ Wd.t()
    dG, dU = dF * u * slope, dF * a
    m = lambda p, q: p.abs() @ q.abs()
    return {"Y": (F @ Wd, m(F, Wd)), "dX": (dG @ Wg.t() + dU @ Wu.t(), m(dG, Wg.t()) + m(dU, Wu.t())), "dWg": (X.t() @ dG, m(X.t(), dG)),
            "dWu": (X.t() @ dU, m(X.t(), dU)), "dWd": (F.t() @ dY, m(F.t(), dY))}


def check(got, want):
    for name, x in got.items():
        value, size = want[name]
        err = (x.double() - value).abs()
        bound = 1.1 * H * size + (H * value.abs() if x.dtype == torch.bfloat16 else 0)
        assert bool((err <= bound).all()), (name, float((err - bound).max()))
        if x.numel() > 10000:
            assert float(err.norm()) <= 2 * H * float(value.norm()), (name, float(err.norm() / value.norm()))


def both(X, dY, W, name, bf16_grads):
    Y = bpt.bpt_gated_ffn_fwd(X, *W, activation=name)
    return dict(zip(("Y", "dX", "dWg", "dWu", "dWd"), (Y,) + bpt.bpt_gated_ffn_bwd(X, *W, dY, activation=name, bf16_grads=bf16_grads)))


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8, 9, 16, 17, 33, 64, 65, 127, 130, 300])
@pytest.mark.parametrize("d,f", [(8, 8), (64, 72), (72, 136), (200, 264), (512, 1368)])
def test_few_rows_and_odd_widths(rows, d, f):
    name = ("silu", "gelu", "relu")[(rows + d) % 3]
    print("gated ffn", rows, d, f, name, flush=True)
    X, dY, W = make(rows, d, f, rows + d + f, gap=8 * (rows % 2))
    check(both(X, dY, W, name, rows % 2 == 0), formulas(X, dY, W, name))


@pytest.mark.parametrize("rows,d,f,name", [(1023, 512, 1368, "silu"), (4099, 264, 1608, "gelu"), (8191, 512, 2048, "relu"),
                                           (16385, 520, 264, "silu"), (2049, 2048, 1032, "gelu"), (70000, 64, 128, "silu"),
                                           (257, 4096, 2056, "silu"), (600, 128, 20000, "relu")])
def test_many_rows_and_wide_blocks(rows, d, f, name):
    print("gated ffn", rows, d, f, name, flush=True)
    X, dY, W = make(rows, d, f, rows + d + f)
    check(both(X, dY, W, name, True), formulas(X, dY, W, name))


def test_rows_between_others_and_no_rows():
    for rows in (1, 7, 200):
        X, dY, W = make(rows, 128, 264, rows, gap=16)
        frame = torch.full((rows + 2, 144), 5.0, dtype=torch.bfloat16, device="cuda")
        Y = bpt.bpt_gated_ffn_fwd(X, *W, out=frame[1:rows + 1, :128])
        check({"Y": Y}, formulas(X, dY, W, "silu"))
        Y.fill_(5.0)
        assert bool((frame == 5.0).all())       # the rows behind the last, and the gaps, as they were
    X, dY, W = make(1, 128, 264, 1)
    got = both(X[:0], dY[:0], W, "silu", False)
    assert got["Y"].shape == (0, 128) and all(bool((got[k] == 0).all()) for k in ("dWg", "dWu", "dWd"))


def test_a_row_that_is_not_finite_stays_alone():
    for rows in (3, 40, 9000):
        X, dY, W = make(rows, 192, 520, rows)
        want = bpt.bpt_gated_ffn_fwd(X, *W)
        X[1, 5] = float("nan")
        X[rows - 1, 0] = float("inf")
        got = bpt.bpt_gated_ffn_fwd(X, *W)
        rest = torch.ones(rows, dtype=torch.bool, device="cuda")
        rest[[1, rows - 1]] = False
        assert torch.equal(got[rest], want[rest]) and bool(torch.isnan(got[1]).all())
        dX = bpt.bpt_gated_ffn_bwd(X, *W, dY)[0]
        assert bool(torch.isfinite(dX[rest]).all())


def test_large_values_of_the_activations():
    # gates far from zero: exp overflows on one side, the slope is 0 or 1 on the other
    X, dY, W = make(64, 64, 128, 3)
    W[0] *= 200
    for name in ("silu", "gelu", "relu"):
        got = both(X, dY, W, name, False)
        assert all(bool(torch.isfinite(v).all()) for v in got.values())
        check(got, formulas(X, dY, W, name))


def test_gradient_written_over_its_input():
    import ctypes
    X, dY, W = make(300, 256, 520, 8)
    want = formulas(X, dY, W, "silu")
    dY, X = dY.contiguous(), X.contiguous()
    s = bpt.BptGatedFfn(300, 256, 520, bpt.BPT_BF16, 0, 256, bpt.BPT_F32)
    L = bpt.load_library()
    need = L.bpt_gated_ffn_bwd_workspace(ctypes.byref(s))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    grads = [torch.empty(w.shape, device="cuda") for w in W]
    assert L.bpt_gated_ffn_bwd(ctypes.byref(s), X.data_ptr(), *[w.data_ptr() for w in W], dY.data_ptr(), dY.data_ptr(),
                               *[g.data_ptr() for g in grads], ws.data_ptr(), need, int(torch.cuda.current_stream().cuda_stream)) == 0
    check(dict(zip(("dX", "dWg", "dWu", "dWd"), [dY] + grads)), want)


def test_gradients_against_differences():
    # the formulas' slope along a random direction; the gradients are off it by the roundings of the module docstring, which are of
    # random sign over the tensor: 4 * 2^-8 of the 2-norms' product is far above them and far below a wrong term
    X, dY, W = make(40, 64, 136, 5)
    for name in ("silu", "gelu"):
        got = both(X, dY, W, name, False)
        inputs = [X.double(), *[w.double() for w in W]]
        for i, key in enumerate(("dX", "dWg", "dWu", "dWd")):
            v = torch.randn(inputs[i].shape, generator=torch.Generator().manual_seed(i)).cuda().double()
            step = 2.0 ** -12

            def value(sign):
                p = list(inputs)
                p[i] = p[i] + sign * step * v
                return float((((act(p[0] @ p[1], name)[0] * (p[0] @ p[2])) @ p[3]) * dY.double()).sum())

            slope = (value(1) - value(-1)) / (2 * step)
            g = got[key].double()
            assert abs(slope - float((g * v).sum())) <= 4 * H * float(g.norm() * v.norm()) + 1e-3, (name, key)


def test_results_are_the_same_twice_and_in_a_replayed_graph():
    for rows in (1, 40, 5000):
        X, dY, W = make(rows, 256, 520, rows)
        want = both(X, dY, W, "silu", True)
        assert all(torch.equal(v, want[k]) for k, v in both(X, dY, W, "silu", True).items())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            both(X, dY, W, "silu", True)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                got = both(X, dY, W, "silu", True)
        torch.cuda.synchronize()
        for _ in range(3):
            for v in got.values():
                v.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(want[k], got[k]) for k in want)
            assert torch.equal(bpt.bpt_gated_ffn_fwd(X, *W), want["Y"])


@pytest.mark.parametrize("rows", [1, 16, 33])
def test_few_rows_of_a_wide_block(rows):
    # the hidden axis of the down product is cut for these: its parts are summed afterwards
    X, dY, W = make(rows, 2048, 5464, rows)
    check(both(X, dY, W, "silu", False), formulas(X, dY, W, "silu"))


@pytest.mark.parametrize("rows,d,f,name", [(2000, 512, 1368, "silu"), (1858, 1344, 744, "gelu"), (3383, 1152, 432, "silu"), (4000, 512, 1368, "silu"),
                                           (700, 1032, 2744, "gelu")])
def test_gradients_of_middle_sizes(rows, d, f, name):
    # dX and the weights' gradients share a launch, in tiles of different sizes
    print("gated ffn", rows, d, f, name, flush=True)
    X, dY, W = make(rows, d, f, rows + d + f)
    check(both(X, dY, W, name, rows % 2 == 0), formulas(X, dY, W, name))


@pytest.mark.parametrize("rows", [5, 300, 4000])
def test_gradient_written_over_the_rows(rows):
    import ctypes
    X, dY, W = make(rows, 256, 520, 9)
    want = formulas(X, dY, W, "silu")
    dY, X = dY.contiguous(), X.contiguous()
    s = bpt.BptGatedFfn(rows, 256, 520, bpt.BPT_BF16, 0, 256, bpt.BPT_F32)
    L = bpt.load_library()
    need = L.bpt_gated_ffn_bwd_workspace(ctypes.byref(s))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    grads = [torch.empty(w.shape, device="cuda") for w in W]
    assert L.bpt_gated_ffn_bwd(ctypes.byref(s), X.data_ptr(), *[w.data_ptr() for w in W], dY.data_ptr(), X.data_ptr(),
                               *[g.data_ptr() for g in grads], ws.data_ptr(), need, int(torch.cuda.current_stream().cuda_stream)) == 0
    check(dict(zip(("dX", "dWg", "dWu", "dWd"), [X] + grads)), want)


def test_rows_far_into_memory():
    # rows and hidden rows whose elements lie more than 2^31 apart.  The partial sums over 2.2e6 rows of values of random sign stay
    # below 2^-7 of the product of magnitudes, so that fp32 adds less than 2.2e6 * 2^-24 * 2^-7 / 8 of it (8 of 16 k to a rounding at
    # least): 0.04 * 2^-8, within the docstring's 0.1
    rows, d, f = 2200000, 64, 1032
    X, dY, W = make(rows, d, f, 12, gap=960)
    got = both(X, dY, W, "silu", False)
    want = {}
    for first in range(0, rows, 200000):
        part = formulas(X[first:first + 200000], dY[first:first + 200000], W, "silu")
        check({k: got[k][first:first + 200000] for k in ("Y", "dX")}, part)
        for k in ("dWg", "dWu", "dWd"):
            want[k] = part[k] if k not in want else tuple(a + b for a, b in zip(want[k], part[k]))
    check({k: got[k] for k in want}, want)


def test_rows_beside_one_that_is_not_finite_keep_their_bits():
    # forward and backward, against the calls before anything was poisoned (the weights' gradients take all rows in)
    for rows in (3, 40, 300, 9000):
        X, dY, W = make(rows, 192, 520, rows)
        want = both(X, dY, W, "gelu", False)
        for which, value in ((X, float("nan")), (dY, float("inf"))):
            kept = which[1].clone()
            which[1, 5] = value
            got = both(X, dY, W, "gelu", False)
            which[1] = kept
            rest = torch.arange(rows, device="cuda") != 1
            for k in ("Y", "dX"):
                assert torch.equal(got[k][rest], want[k][rest]), (rows, k)
            assert not bool(torch.isfinite(got["dX"][1]).any())
