"""The block's operators on layouts that torch hands over in passing: axes of one entry with strides of their own, slices."""
import pytest
import torch

from paper_1911_04070_amd import binding as bpt
from test_gpu_rotary import check as check_rotary, make as make_heads, reference as turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(2, 1, 37), (3, 4, 1), (1, 3, 5), (4, 1, 1), (5000, 3, 1), (1, 1, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotary_with_unit_axes(shape, dtype):
    # Q, K and their gradients in every pair of layouts that are one and the same to torch or differ in truth (tolerances: test_gpu_rotary)
    B, H, N = shape
    pos = torch.arange(N, dtype=torch.float32, device="cuda") * 2 + 5
    for of_q, of_k in (("heads", "nodes"), ("nodes", "heads")):
        print("rotary", shape, dtype, of_q, of_k, flush=True)
        Q, K = make_heads(B, H, N, dtype, of_q, 1), make_heads(B, H, N, dtype, of_k, 2)
        if bpt._lie_alike(Q, K):
            for x, y in zip((Q, K), bpt.bpt_rotary(Q, K, pos)):
                check_rotary(y, *turned(x, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, False), dtype)
        Q, K = (make_heads(B, H, N, dtype, "heads", s).requires_grad_() for s in (1, 2))
        gq, gk = make_heads(B, H, N, dtype, of_q, 3), make_heads(B, H, N, dtype, of_k, 4)
        for g, d in zip((gq, gk), torch.autograd.grad(bpt.rotary(Q, K, pos), (Q, K), (gq, gk))):
            check_rotary(d, *turned(g, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, True), dtype)


def test_rows_with_unit_axes():
    # [1, rows, d] against [rows, 1, d] turned round: the same rows in the same places
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=gen).bfloat16().cuda()
    rows, d, f = 37, 64, 136
    W = [r(d, f) * 0.125, r(d, f) * 0.125, r(f, d) * 0.0625]
    x, b, dy = r(rows, d), r(rows, d), r(rows, d)
    dense = lambda t: t.view(1, rows, d)
    turned_round = lambda t: t.view(rows, 1, d).transpose(0, 1)

    def work(place, other):
        X, B = place(x).requires_grad_(), other(b).requires_grad_()
        y, h = bpt.residual_norm(X, B)
        Y = bpt.gated_ffn(X, *W)
        return (y, h, Y) + torch.autograd.grad((y, h, Y), (X, B), (other(dy), place(dy), other(dy)))

    want = work(dense, dense)
    for place, other in ((dense, turned_round), (turned_round, dense), (turned_round, turned_round)):
        assert all(torch.equal(a, w) for a, w in zip(work(place, other), want))


@pytest.mark.parametrize("rows,d,f", [(1, 64, 72), (5, 512, 1368), (40, 136, 264), (300, 512, 520), (4001, 264, 1032)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_each_tensor_lies_as_it_likes(rows, d, f, dtype):
    # every tensor of a call in a layout of its own against all of them dense: the same bits; what lies around results is left alone
    print("layouts", rows, d, f, dtype, flush=True)
    gen = torch.Generator().manual_seed(rows + d)
    r = lambda *s: torch.randn(s, generator=gen)
    x, b, dy, dh = (r(rows, 1, d).to(dtype).cuda() for _ in range(4))
    gate = r(-(-rows // 3), d).to(dtype).cuda()
    gain, bias = (1 + 0.1 * r(d)).cuda(), (0.1 * r(d)).cuda()
    how = dict(post="rms", pre="layer", post_gain=gain, post_bias=bias, pre_gain=gain, pre_bias=bias, gate_rows=3, residual_scale=0.75)
    W = [(r(d, f) * d ** -0.5).bfloat16().cuda(), (r(d, f) * d ** -0.5).bfloat16().cuda(), (r(f, d) * f ** -0.5).bfloat16().cuda()]

    def apart(t, before, after):      # the rows of t in the middle of longer sequences
        frame = torch.full((rows, before + 1 + after, d), 9.0, dtype=t.dtype, device="cuda")
        frame[:, before:before + 1] = t
        return frame[:, before:before + 1]

    def work(x, b, dy, dh):
        y, h, stats = bpt.bpt_residual_norm_fwd(x, b, gate, want_stats=True, **how)
        got = [y, h] + [v for _, v in sorted(bpt.bpt_residual_norm_bwd(x, b, gate, stats, dy, dh, **how).items())]
        if dtype == torch.bfloat16:
            got += [bpt.bpt_gated_ffn_fwd(x, *W), *bpt.bpt_gated_ffn_bwd(x, *W, dy)]
        return got

    want = work(x, b, dy, dh)
    for place in ((6, 0, 0, 0), (0, 3, 0, 0), (0, 0, 5, 0), (0, 0, 0, 2), (2, 2, 2, 2), (1, 2, 3, 3), (3, 0, 2, 1)):
        tensors = [apart(t, n, n // 2) if n else t for t, n in zip((x, b, dy, dh), place)]
        got = work(*tensors)
        assert all(torch.equal(a, w) for a, w in zip(got, want)), place
        assert all(t.is_contiguous() for t in got)
    if dtype == torch.bfloat16:
        frame = torch.full((rows, 3, d), 9.0, dtype=dtype, device="cuda")
        Y = bpt.bpt_gated_ffn_fwd(apart(x, 6, 0), *W, out=frame[:, 1:2])
        assert torch.equal(Y, bpt.bpt_gated_ffn_fwd(x, *W))
        assert bool((frame[:, ::2] == 9.0).all())


def test_the_last_rows_of_long_sequences():
    # a decoding step on what the sequences' last tokens left: 32 rows, 2^22 elements apart, beside a dense branch
    states = torch.zeros((32, 8192, 512), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(2)
    last = states[:, -1:]
    last.copy_(torch.randn((32, 1, 512), generator=gen))
    branch = torch.randn((32, 1, 512), generator=gen).bfloat16().cuda()
    before = torch.cuda.memory_allocated()
    y, h = bpt.bpt_residual_norm_fwd(last, branch)
    assert torch.cuda.memory_allocated() - before <= 2 * max(32 * 512 * 2, 512) + 1024
    want = bpt.bpt_residual_norm_fwd(last.contiguous(), branch)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    # the same rows through the feed-forward block, forward and backward
    W = [(torch.randn(s, generator=gen) * s[0] ** -0.5).bfloat16().cuda().requires_grad_() for s in ((512, 264), (512, 264), (264, 512))]
    leaves = [last.detach().requires_grad_(), last.contiguous().requires_grad_()]
    got, want = ([Y] + list(torch.autograd.grad(Y, [x] + W, branch)) for x in leaves for Y in (bpt.gated_ffn(x, *W),))
    assert all(torch.equal(a, w) for a, w in zip(got, want))
    assert torch.equal(bpt.bpt_gated_ffn_fwd(last, *[w.detach() for w in W], out=last), want[0]) and torch.equal(last, want[0])
    assert not bool(states[:, :-1].any())


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_positions_of_a_graph_on_another_device_are_refused():
    g = bpt.bpt_build_batch_graph(64, 2, True, [5, 64])
    with torch.cuda.device(1), pytest.raises(bpt.BptError):
        bpt.bpt_node_positions(g)
    assert bpt.bpt_node_positions(g).shape == (g.num_nodes,)
    g.destroy()
