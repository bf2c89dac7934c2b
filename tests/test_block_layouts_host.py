"""What the binding hands to the block's operators for tensors of any layout, on the host: the library is a stand-in that writes down
the arguments it is called with."""
import ctypes

import pytest
import torch

from paper_1911_04070_amd import binding as bpt


class Recorder:
    """Answers every call with 0 and keeps (name, arguments); structures passed by reference are copied."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            kept = []
            for a in args:
                a = getattr(a, "_obj", a)
                kept.append(type(a).from_buffer_copy(a) if isinstance(a, ctypes.Structure) else a)
            self.calls.append((name, kept))
            return 0
        return call


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(bpt, "load_library", lambda: r)
    monkeypatch.setattr(bpt, "_on_device", lambda x, what: x.device)
    monkeypatch.setattr(bpt, "_raw_stream", lambda index: 0)
    return r


def heads(B, H, N):
    return torch.zeros((B, H, N, 64))


def nodes(B, H, N):
    return torch.zeros((B, N, H, 64)).permute(0, 2, 1, 3)


UNIT_AXES = [(2, 1, 37), (3, 4, 1), (1, 3, 5), (2, 1, 1), (1, 1, 9), (1, 1, 1)]


@pytest.mark.parametrize("shape", UNIT_AXES)
def test_rotary_takes_unit_axes_of_any_stride(recorder, shape):
    # what torch counts as one layout, whatever it has set the strides of axes of one entry to
    B, H, N = shape
    like = [f(*shape) for f in (heads, nodes)]
    like += [x.as_strided(x.shape, [12345 if n == 1 else s for n, s in zip(x.shape, x.stride())]) for x in like]
    pos = torch.zeros(N)
    for Q in like:
        for K in like:
            if bpt._head_strides(Q) != bpt._head_strides(K):
                continue
            Qr, Kr = bpt.bpt_rotary(Q, K, pos)
            bpt.bpt_rotary(Q, K, pos, out=(Qr, Kr))
            bpt.bpt_rotary(Q, K, pos, out=(Q, K))
            assert Qr.shape == Kr.shape == Q.shape
            assert bpt._head_strides(Qr) == bpt._head_strides(Kr)


@pytest.mark.parametrize("shape", UNIT_AXES + [(2, 3, 5)])
def test_rotary_gradients_with_unit_axes(recorder, shape):
    B, H, N = shape
    for f in (heads, nodes):
        for of_q in (heads, nodes):
            for of_k in (heads, nodes):
                Q, K = f(*shape).requires_grad_(), f(*shape).requires_grad_()
                got = torch.autograd.grad(bpt.rotary(Q, K, torch.zeros(N)), (Q, K), (of_q(*shape), of_k(*shape)))
                assert all(g.shape == Q.shape for g in got)


def test_rotary_gradients_are_turned_as_they_lie(recorder):
    # different layouts of dQ and dK: a call each, nothing copied
    Q, K = heads(2, 3, 5).requires_grad_(), heads(2, 3, 5).requires_grad_()
    out = bpt.rotary(Q, K, torch.zeros(5))
    gq, gk = heads(2, 3, 5), nodes(2, 3, 5)
    del recorder.calls[:]
    torch.autograd.grad(out, (Q, K), (gq, gk))
    assert [c[1][3] for c in recorder.calls] == [gq.data_ptr(), gk.data_ptr()]
    assert all(c[1][4] is None and c[1][0].inverse for c in recorder.calls)


def test_rotary_refuses_layouts_that_differ(recorder):
    with pytest.raises(ValueError, match="share"):
        bpt.bpt_rotary(heads(2, 3, 5), nodes(2, 3, 5), torch.zeros(5))
    with pytest.raises(ValueError, match="results"):
        bpt.bpt_rotary(heads(2, 3, 5), heads(2, 3, 5), torch.zeros(5), out=(heads(2, 3, 5), nodes(2, 3, 5)))


def test_the_library_does_not_look_at_strides_of_unit_axes():
    # answered on the host: B = 1, H = 1 and N = 1 with strides that would be refused
    L = bpt.load_library()
    good = dict(B=2, H=3, N=5, D=64, dtype=0, rot=64, stride_b=960, stride_h=320, stride_n=64, out_stride_b=960, out_stride_h=320, out_stride_n=64)

    def call(**kw):
        s = bpt.BptRotary()
        for k, v in {**good, **kw}.items():
            setattr(s, k, v)
        return L.bpt_rotary(ctypes.byref(s), None, 0, None, None, None, None, None)

    for axis, count in (("b", "B"), ("h", "H"), ("n", "N")):
        odd = {"stride_" + axis: 7, "out_stride_" + axis: -3}
        assert call(**odd) == bpt.BPT_ERR_INVALID_ARG
        # no heads or no rows: nothing to do, and nothing refused
        other = "H" if count != "H" else "N"
        assert call(**{count: 1, other: 0}, **odd) == bpt.BPT_OK


def one_layout(rows=6, d=64, dtype=torch.bfloat16):
    """[1, rows, d] tensors that lie alike, with different strides of the axis of one entry"""
    x = torch.zeros((1, rows, d), dtype=dtype)
    return [x, torch.zeros((rows, 1, d), dtype=dtype).transpose(0, 1), x.as_strided(x.shape, (7, d, 1))]


def test_rows_with_unit_axes(recorder):
    d = 64
    W = [torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((128, d), dtype=torch.bfloat16)]
    stats = torch.zeros((6, 4))
    for a in one_layout():
        for b in one_layout():
            y, h = bpt.bpt_residual_norm_fwd(a, b)
            assert y.shape == h.shape == a.shape
            got = bpt.bpt_residual_norm_bwd(a, b, None, stats, b, a)
            assert got["dx"].shape == got["d_branch"].shape == a.shape
            assert bpt.bpt_gated_ffn_fwd(a, *W, out=b) is b
            assert bpt.bpt_gated_ffn_bwd(a, *W, b)[0].shape == a.shape


def test_rows_that_differ_are_refused(recorder):
    x = torch.zeros((1, 6, 64), dtype=torch.bfloat16)
    for other in (x[:, :5], x.float(), torch.zeros((6, 1, 64), dtype=torch.bfloat16), torch.zeros((1, 6, 128), dtype=torch.bfloat16)[..., ::2],
                  x[:, :1].expand(1, 6, 64)):
        with pytest.raises(ValueError):
            bpt.bpt_residual_norm_fwd(x, other)


def storage(t):
    return t.untyped_storage().nbytes() // t.element_size()


def slices(d=64, dtype=torch.bfloat16):
    """[4, 1, d] tensors: dense, the last rows of longer sequences, and a part of wider rows"""
    return [torch.zeros((4, 1, d), dtype=dtype), torch.zeros((4, 7, d), dtype=dtype)[:, -1:], torch.zeros((4, 1, 3 * d), dtype=dtype)[..., d:2 * d]]


def test_results_take_the_memory_of_their_own_rows(recorder):
    d, f = 64, 128
    W = [torch.zeros((d, f), dtype=torch.bfloat16), torch.zeros((d, f), dtype=torch.bfloat16), torch.zeros((f, d), dtype=torch.bfloat16)]
    stats = torch.zeros((4, 4))
    for x in slices():
        results = list(bpt.bpt_residual_norm_fwd(x, x)) + list(bpt.bpt_residual_norm_bwd(x, x, None, stats, x, x).values())
        results += [bpt.bpt_gated_ffn_fwd(x, *W), bpt.bpt_gated_ffn_bwd(x, *W, x)[0]]
        leaf = x.requires_grad_()
        for out in bpt.residual_norm(leaf, leaf) + (bpt.gated_ffn(leaf, *W),):
            results += [out, torch.autograd.grad(out, leaf, torch.zeros((4, 7, d), dtype=x.dtype)[:, 2:3], retain_graph=True)[0]]
        assert len(results) == 12
        for t in results:
            assert t.shape == x.shape and t.is_contiguous() and storage(t) == x.numel()


def test_rows_lie_where_their_tensors_say(recorder):
    # each tensor's own distance of rows goes into the call; contiguous tensors need none
    stats = torch.zeros((4, 4))
    W = [torch.zeros((64, 128), dtype=torch.bfloat16), torch.zeros((64, 128), dtype=torch.bfloat16), torch.zeros((128, 64), dtype=torch.bfloat16)]
    apart = {0: 64, 1: 448, 2: 192}

    def strides():
        name, args = [c for c in recorder.calls if c[0].endswith("_strided")][-1]
        assert args[0].stride == 64
        return None if args[1] is None else (args[1].x, args[1].branch, args[1].out, args[1].grad)

    for i, x in enumerate(slices()):
        for j, b in enumerate(slices()):
            bpt.bpt_residual_norm_fwd(x, b)
            assert strides() == (None if i == j == 0 else (apart[i], apart[j], 64, 64))
            bpt.bpt_gated_ffn_fwd(x, *W, out=b)
            assert strides() == (None if i == j == 0 else (apart[i], 64, apart[j], 64))
            bpt.bpt_gated_ffn_bwd(x, *W, b)
            assert strides() == (None if i == j == 0 else (apart[i], 64, 64, apart[j]))
            for k, g in enumerate(slices()):
                bpt.bpt_residual_norm_bwd(x, b, None, stats, g, g)
                assert strides() == (None if i == j == k == 0 else (apart[i], apart[j], 64, apart[k]))
            # dy and dh lie differently: both are made contiguous
            bpt.bpt_residual_norm_bwd(x, x, None, stats, x, b)
            assert strides() == (None if i == 0 else (apart[i], apart[i], 64, apart[i] if i == j else 64))


def test_strided_calls_refuse_what_they_cannot_read():
    L = bpt.load_library()
    INVALID = bpt.BPT_ERR_INVALID_ARG
    P = [4096 * (i + 1) for i in range(20)]
    norm = bpt.BptResidualNorm(10, 64, bpt.BPT_BF16, 64, 0, 2, 0, 1.0, 0.0)
    ffn = bpt.BptGatedFfn(10, 64, 128, bpt.BPT_BF16, 0, 64, bpt.BPT_F32)
    grads = bpt.BptResidualNormGrads()

    # (only calls that are refused are made: the pointers are made-up numbers)
    def call(which, s, y=P[6], dx=P[9], dX=P[6]):
        s = ctypes.byref(bpt.BptRowStrides(*s))
        if which == "norm":
            return L.bpt_residual_norm_fwd_strided(ctypes.byref(norm), s, P[0], P[1], None, None, None, None, None, y, P[7], None, None)
        if which == "norm backward":
            return L.bpt_residual_norm_bwd_strided(ctypes.byref(norm), s, P[0], P[1], None, None, None, None, None, P[6], P[7], P[8], dx, P[10],
                                                   ctypes.byref(grads), P[15], 1 << 30, None)
        if which == "ffn":
            return L.bpt_gated_ffn_fwd_strided(ctypes.byref(ffn), s, *P[:4], y, P[10], 1 << 40, None)
        return L.bpt_gated_ffn_bwd_strided(ctypes.byref(ffn), s, *P[:5], dX, *P[7:10], P[10], 1 << 40, None)

    every = ("norm", "norm backward", "ffn", "ffn backward")
    readers = (every, every[:2], every, ("norm backward", "ffn backward"))   # of x, branch, out, grad
    for at, which in enumerate(readers):
        for bad in (56, 68, 0, -64, 1 << 41, 1 << 20):
            s = [64] * 4
            s[at] = bad
            for w in which:
                if bad != 1 << 20 or w.startswith("ffn"):    # (the feed-forward block's offsets within a tile have 32 bits)
                    assert call(w, s) == INVALID, (w, at, bad)
    # a result over an input of another distance
    for y in P[:2]:
        assert call("norm", (64, 64, 72, 64), y=y) == INVALID
    for dx in P[7:9]:
        assert call("norm backward", (64, 64, 72, 64), dx=dx) == INVALID
    for dX in (P[0], P[4]):
        assert call("ffn backward", (64, 64, 72, 64), dX=dX) == INVALID


def test_rows_too_far_apart_for_the_products_are_copied_together(recorder):
    d = 64
    W = [torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((128, d), dtype=torch.bfloat16)]
    for tokens, strides in (((1 << 20) // d - 1, (1 << 20) - d), ((1 << 20) // d, None), ((1 << 20) // d + 3, None)):
        x = torch.zeros((3, tokens, d), dtype=torch.bfloat16)[:, -1:]
        del recorder.calls[:]
        assert bpt.bpt_gated_ffn_fwd(x, *W).shape == x.shape
        assert bpt.bpt_gated_ffn_fwd(x, *W, out=x) is x
        bpt.bpt_gated_ffn_bwd(x, *W, x)
        for name, args in recorder.calls:
            if name.endswith("_strided"):
                assert (args[1] is None) == (strides is None) and (strides is None or args[1].x == strides)
                assert (args[2] == x.data_ptr()) == (strides is not None)


def test_a_workspace_of_the_callers_is_memory_of_the_device(recorder):
    d = 64
    W = [torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((d, 128), dtype=torch.bfloat16), torch.zeros((128, d), dtype=torch.bfloat16)]
    x = torch.zeros((4, d), dtype=torch.bfloat16)
    calls = (lambda ws: bpt.bpt_gated_ffn_fwd(x, *W, workspace=ws), lambda ws: bpt.bpt_gated_ffn_bwd(x, *W, x, workspace=ws))
    for call in calls:
        for ws in (torch.empty(1 << 20, dtype=torch.uint8, device="meta"),        # of another device
                   torch.zeros(1, dtype=torch.uint8).expand(1 << 20),             # one byte, counted a million times
                   torch.zeros(1 << 21, dtype=torch.uint8)[::2]):                 # bytes in between that are not the workspace's
            del recorder.calls[:]
            with pytest.raises(ValueError, match="workspace"):
                call(ws)
            assert not any(name.endswith("_strided") for name, _ in recorder.calls)
        ws = torch.empty((16, 100), dtype=torch.float32)
        call(ws)
        assert recorder.calls[-1][1][-3:-1] == [ws.data_ptr(), 6400]
