"""Refusals of the block's operators, on the host: every call here is answered before anything touches a device (the pointers are
made-up numbers)."""
import ctypes

import pytest
import torch

from paper_1911_04070_amd import binding as bpt

OK, INVALID, UNSUPPORTED = bpt.BPT_OK, bpt.BPT_ERR_INVALID_ARG, bpt.BPT_ERR_UNSUPPORTED
P = [4096 * (i + 1) for i in range(20)]
SIZE_MAX = 2 ** 64 - 1


def struct(cls, usual, **kw):
    s = cls()
    for k, v in {**usual, **kw}.items():
        setattr(s, k, v)
    return s


ROTARY = dict(B=2, H=3, N=5, D=64, dtype=0, stride_b=960, stride_h=320, stride_n=64, out_stride_b=960, out_stride_h=320,
              out_stride_n=64, rot=64)


def rotary(ptrs=None, pos_stride=0, **kw):
    pos, Q, K, Qr, Kr = ptrs if ptrs else P[:5]
    return bpt.load_library().bpt_rotary(ctypes.byref(struct(bpt.BptRotary, ROTARY, **kw)), pos, pos_stride, Q, K, Qr, Kr, None)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(bpt.BptRotary) == 128 and bpt.BptRotary.stride_b.offset == 24 and bpt.BptRotary.rot.offset == 72
    assert bpt.BptRotary.base.offset == 88
    assert ctypes.sizeof(bpt.BptResidualNorm) == 48 and bpt.BptResidualNorm.gate_rows.offset == 32
    assert ctypes.sizeof(bpt.BptGatedFfn) == 40 and bpt.BptGatedFfn.stride.offset == 24
    assert ctypes.sizeof(bpt.BptResidualNormGrads) == 40


@pytest.mark.parametrize("kw,code", [
    (dict(D=32), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(rot=0), INVALID), (dict(rot=7), INVALID), (dict(rot=66), INVALID),
    (dict(B=-1), INVALID), (dict(stride_n=-64), INVALID), (dict(stride_n=68), INVALID), (dict(out_stride_n=32), INVALID),
    (dict(out_stride_h=0), INVALID), (dict(out_stride_b=480), INVALID), (dict(out_stride_n=128), INVALID), (dict(pos_stride=-1), INVALID),
    (dict(context=-1.0), INVALID), (dict(low=4.0, high=2.0), INVALID), (dict(factor=float("inf")), INVALID),
    (dict(base=float("nan")), INVALID), (dict(factor=float("nan")), INVALID), (dict(B=1 << 14, N=1 << 14, out_stride_b=1 << 40), UNSUPPORTED), (dict(H=70000), UNSUPPORTED),
])
def test_rotary_refuses(kw, code):
    assert rotary(**kw) == code


def test_rotary_refuses_pointers():
    assert bpt.load_library().bpt_rotary(None, P[0], 0, P[1], P[2], P[3], P[4], None) == INVALID
    for i in range(5):
        gone = list(P[:5])
        gone[i] = None
        assert rotary(gone) == INVALID
        off = list(P[:5])
        off[i] += 8 if i else 2      # positions may start at any fp32
        assert rotary(off) == INVALID
    assert rotary([P[0], P[1], P[2], P[3], P[3]]) == INVALID            # both results in one place
    assert rotary([P[0], P[1], P[2], P[2], P[4]]) == INVALID            # Q's result over K
    assert rotary([P[0], P[1], P[2], P[1], P[4]], out_stride_b=1920) == INVALID   # in place with other strides
    for kw in (dict(B=0), dict(H=0), dict(N=0)):
        assert rotary([None] * 5, **kw) == OK
    assert bpt.load_library().bpt_node_positions(None, P[0], None) == INVALID


NORM = dict(rows=10, d=64, dtype=1, stride=64, post=2, pre=1, gate_rows=0, residual_scale=1.0, eps=0.0)


def norm_fwd(x=P[0], branch=P[1], gate=None, pg=P[2], pb=P[3], qg=P[4], qb=P[5], y=P[6], h=P[7], stats=P[8], **kw):
    s = struct(bpt.BptResidualNorm, NORM, **kw)
    return bpt.load_library().bpt_residual_norm_fwd(ctypes.byref(s), x, branch, gate, pg, pb, qg, qb, y, h, stats, None)


def norm_bwd(x=P[0], branch=P[1], gate=None, pg=P[2], pb=P[3], qg=P[4], qb=P[5], stats=P[6], dy=P[7], dh=P[8], dx=P[9], db=P[10],
             grads=(None, P[11], P[12], P[13], P[14]), ws=P[15], ws_bytes=1 << 30, **kw):
    s = struct(bpt.BptResidualNorm, NORM, **kw)
    g = bpt.BptResidualNormGrads(*grads)
    return bpt.load_library().bpt_residual_norm_bwd(ctypes.byref(s), x, branch, gate, pg, pb, qg, qb, stats, dy, dh, dx, db,
                                                    ctypes.byref(g), ws, ws_bytes, None)


BAD_NORMS = [(dict(rows=-1), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(d=12), UNSUPPORTED),
             (dict(d=0), UNSUPPORTED), (dict(d=4104, stride=4104), UNSUPPORTED), (dict(stride=56), INVALID), (dict(stride=68), INVALID),
             (dict(post=3), INVALID), (dict(pre=-1), INVALID), (dict(gate_rows=-1), INVALID), (dict(gate_rows=5), INVALID),
             (dict(residual_scale=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x=None), INVALID),
             (dict(branch=None), INVALID), (dict(gate=P[16]), INVALID), (dict(post=0), INVALID), (dict(pg=P[2] + 4), INVALID),
             (dict(x=P[0] + 2), INVALID)]


@pytest.mark.parametrize("kw,code", BAD_NORMS + [(dict(h=None), INVALID), (dict(y=P[6], h=P[6]), INVALID), (dict(stats=P[8] + 8), INVALID),
                                                 (dict(pre=0, qg=None, qb=None), INVALID),
                                                 (dict(pre=0, qg=None, qb=None, h=None, y=None), INVALID)])
def test_residual_norm_refuses(kw, code):
    assert norm_fwd(**kw) == code


@pytest.mark.parametrize("kw,code", BAD_NORMS + [
    (dict(stats=None), INVALID), (dict(dy=None, dh=None), INVALID), (dict(dx=None), INVALID), (dict(db=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws_bytes=100), INVALID), (dict(dx=P[9], db=P[9]), INVALID), (dict(grads=(P[16], P[11], P[12], P[13], P[14])), INVALID),
    (dict(grads=(None, None, P[12], P[13], P[14])), INVALID), (dict(grads=(None, P[11], P[12], P[13] + 4, P[14])), INVALID),
    (dict(pre=0, qg=None, qb=None, grads=(None, P[11], P[12], None, None)), INVALID)])   # dh without a norm behind it
def test_residual_norm_backward_refuses(kw, code):
    assert norm_bwd(**kw) == code


def test_residual_norm_of_no_rows_and_its_workspace():
    L = bpt.load_library()
    assert norm_fwd(rows=0, x=None, y=None, h=None) == OK
    assert L.bpt_residual_norm_bwd_workspace(None) == SIZE_MAX
    assert L.bpt_residual_norm_bwd_workspace(ctypes.byref(struct(bpt.BptResidualNorm, NORM, d=12))) == SIZE_MAX
    assert L.bpt_residual_norm_bwd_workspace(ctypes.byref(struct(bpt.BptResidualNorm, NORM, rows=0))) == 0
    for rows in (1, 10, 100000, (1 << 31) - 2):
        for gate_rows in (0, 1, 2, 1000, (1 << 31) - 2):
            need = L.bpt_residual_norm_bwd_workspace(ctypes.byref(struct(bpt.BptResidualNorm, NORM, rows=rows, gate_rows=gate_rows)))
            assert 0 < need < 1 << 30
    assert L.bpt_residual_norm_bwd(None, *[None] * 12, None, None, 0, None) == INVALID


FFN = dict(rows=10, d=64, f=128, dtype=1, activation=0, stride=64, grad_dtype=0)


def ffn(fwd, ptrs=None, ws=P[10], ws_bytes=1 << 40, **kw):
    s = struct(bpt.BptGatedFfn, FFN, **kw)
    L = bpt.load_library()
    if fwd:
        return L.bpt_gated_ffn_fwd(ctypes.byref(s), *(ptrs or P[:5]), ws, ws_bytes, None)
    return L.bpt_gated_ffn_bwd(ctypes.byref(s), *(ptrs or P[:9]), ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED), (dict(d=12), UNSUPPORTED), (dict(d=0), UNSUPPORTED),
    (dict(f=4), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED), (dict(rows=1 << 21, f=65536), UNSUPPORTED), (dict(f=65544), UNSUPPORTED), (dict(stride=56), INVALID), (dict(stride=66), INVALID), (dict(stride=1 << 20), INVALID),
    (dict(activation=3), INVALID), (dict(activation=-1), INVALID), (dict(grad_dtype=2), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=64), INVALID),
    (dict(ws=P[10] + 8), INVALID)])
def test_gated_ffn_refuses(kw, code):
    assert ffn(True, **kw) == code
    assert ffn(False, **kw) == code


def test_gated_ffn_refuses_pointers_and_answers_workspaces():
    L = bpt.load_library()
    for fwd, count in ((True, 5), (False, 9)):
        for i in range(count):
            for value in (None, P[i] + 4):
                ptrs = list(P[:count])
                ptrs[i] = value
                assert ffn(fwd, ptrs) == INVALID
    assert ffn(True, [None] * 5, ws=None, rows=0) == OK
    assert L.bpt_gated_ffn_fwd(None, *[None] * 6, 0, None) == INVALID and L.bpt_gated_ffn_bwd(None, *[None] * 10, 0, None) == INVALID
    for query in (L.bpt_gated_ffn_fwd_workspace, L.bpt_gated_ffn_bwd_workspace):
        assert query(None) == SIZE_MAX
        assert query(ctypes.byref(struct(bpt.BptGatedFfn, FFN, d=12))) == SIZE_MAX
        for rows in (0, 1, 7, 1000, 1 << 20):
            for d, f in ((8, 8), (64, 128), (2048, 8), (8, 65536), (65536, 65536)):
                need = query(ctypes.byref(struct(bpt.BptGatedFfn, FFN, rows=rows, d=d, f=f, stride=d)))
                assert need >= 2 * rows * f or need == SIZE_MAX


def test_the_binding_takes_no_tensors_from_elsewhere():
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="cuda"):
        bpt.bpt_residual_norm_fwd(x, x)
    with pytest.raises(ValueError, match="cuda"):
        bpt.bpt_rotary(x.view(1, 1, 4, 64), None, torch.zeros(4))
    with pytest.raises(ValueError, match="cuda"):
        bpt.bpt_gated_ffn_fwd(x.bfloat16(), x, x, x)


def test_rows_that_lie_evenly_apart():
    base = torch.zeros((4, 6, 24))
    for x, stride in ((base, 24), (base[:, :1], 144), (base[:, -1:], 144), (base[1:3, 2:3], 144), (base[..., :16], 24), (base[:1, ::2], 48),
                      (base[0, 0], 24), (base[:1, :1], 24), (base[:0], 24), (base[:, :0], 24), (base.view(2, 2, 6, 24)[:, :, 5:], 144),
                      (base.view(2, 2, 6, 24)[:, :1, 5:], 288)):
        assert bpt._row_stride(x, "x") == stride, (x.shape, x.stride())
    for x in (base[:, :3], base.transpose(0, 1), base.transpose(1, 2), base[..., ::2], base[:1].expand(4, 6, 24),
              base[:, :1].expand(4, 6, 24), base[0, :1].expand(6, 24)):
        with pytest.raises(ValueError):
            bpt._row_stride(x, "x")


def test_gated_ffn_workspaces_of_every_shape_the_calls_take():
    # refused exactly where a launch would have too many tiles; else room for the hidden activations (three of them backward) and sums
    L = bpt.load_library()
    refused = 0
    for rows in (0, 1, 7, 1000, 8191, 1 << 20, (1 << 23) - 64, 1 << 23):
        for d, f in ((8, 8), (64, 128), (2048, 8), (8, 65536), (4096, 16384), (65536, 65536)):
            tiles = max(-(-rows // 64) * -(-d // 64), -(-rows // 128) * -(-f // 128))
            refused += tiles >= 1 << 23
            for query, hidden in ((L.bpt_gated_ffn_fwd_workspace, 1), (L.bpt_gated_ffn_bwd_workspace, 3)):
                need = query(ctypes.byref(struct(bpt.BptGatedFfn, FFN, rows=rows, d=d, f=f, stride=d)))
                assert (need == SIZE_MAX) == (tiles >= 1 << 23), (rows, d, f)
                # (hidden activations in two parts at most; sums of parts: as many tiles as the device holds at once, 64 MB)
                assert need == SIZE_MAX or hidden * 2 * rows * f <= need <= hidden * 4 * rows * f + (1 << 27)
    assert refused > 0
