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
            bpt.bpt_rotary(Q, K, pos, out=(K, Q))
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
