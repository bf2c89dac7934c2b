"""Rotary positions and node positions against a plain implementation in 64 bits.

Tolerance, for a pair (a, b): the reduced angle is rounded to fp32 as a fraction of a turn of at most 1/2 (error 2^-26 of a
turn, doubled in the argument of sincospi: 2 pi 2^-26 < 0.81 * 2^-23 in the angle), sincospi is good to two units in the last
place (2^-23), each product and the sum round once (2^-24 each): at most 2.9 * 2^-23 (|a| + |b|); 2^-21 (|a| + |b|) is used.
The result is rounded to the tensors' type: 2^-8 relative for bf16, 2^-24 for fp32.
"""
import math

import numpy as np
import pytest
import torch

from paper_1911_04070_amd import binding as bpt

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def make(B, H, N, dtype, layout, seed):
    gen = torch.Generator().manual_seed(seed)
    if layout == "heads":
        x = torch.randn((B, H, N, 64), generator=gen)
    elif layout == "nodes":
        x = torch.randn((B, N, H, 64), generator=gen).permute(0, 2, 1, 3)
    else:   # gaps between rows, heads and batches
        x = torch.randn((B, H + 1, N + 2, 80), generator=gen)[:, :H, 1:N + 1, 8:72]
    return torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda").copy_(x)


def reference(x, pos, rot, interleaved, base, factor, context, low, high, inverse):
    """(result, |a| + |b| of every feature's pair), fp64."""
    x = x.double().cpu()
    i = torch.arange(rot // 2, dtype=torch.float64)
    w = base ** (-2.0 * i / rot)
    keep = ((context * w / (2 * math.pi) - low) / (high - low)).clamp(0, 1) if context else torch.zeros_like(w)
    w = w * (keep + (1 - keep) / factor)
    p = pos.double().cpu()
    t = (p if p.dim() == 2 else p[None]).reshape(-1, 1, x.shape[2], 1) * w * (-1 if inverse else 1)
    first = 2 * torch.arange(rot // 2) if interleaved else torch.arange(rot // 2)
    second = first + 1 if interleaved else first + rot // 2
    y, size = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first] = a * t.cos() - b * t.sin()
    y[..., second] = b * t.cos() + a * t.sin()
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def check(got, want, size, dtype):
    err = (got.double().cpu() - want).abs()
    assert (err <= HALF_STEP[dtype] * want.abs() + 2.0 ** -21 * size).all(), float(err.max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rot", [2, 6, 12, 16, 24, 32, 48, 62, 64])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_parts_of_the_head(dtype, rot, interleaved):
    print("rotary", dtype, rot, interleaved, flush=True)
    for (B, H, N), layout, far in (((1, 1, 1), "heads", 0), ((3, 2, 37), "nodes", 5000), ((2, 5, 130), "gaps", 1 << 20)):
        Q, K = make(B, H, N, dtype, layout, 7 * rot + N), make(B, H, N, dtype, layout, 7 * rot + N + 1)
        pos = (torch.arange(N) + far - 0.5 * (N > 40)).float().cuda()
        for inverse in (False, True):
            got = bpt.bpt_rotary(Q, K, pos, rot=rot, interleaved=interleaved, inverse=inverse)
            for x, y in zip((Q, K), got):
                want, size = reference(x, pos, rot, interleaved, 10000.0, 1.0, 0, 1.0, 32.0, inverse)
                check(y, want, size, dtype)
                assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("factor,context,low,high", [(4.0, 0, 1.0, 32.0), (8.0, 2048, 1.0, 32.0), (2.0, 100, 0.5, 4.0), (0.5, 4096, 1.0, 32.0)])
def test_rotary_for_long_contexts_and_positions_of_each_sequence(factor, context, low, high):
    Q = make(4, 3, 9, torch.float32, "heads", 3)
    pos = torch.tensor([[0.0], [777.0], [(1 << 23) - 20.0], [-5.5]]) + torch.arange(9)
    got, none = bpt.bpt_rotary(Q, None, pos.cuda(), factor=factor, context=context, low=low, high=high, base=500.0)
    assert none is None
    check(got, *reference(Q, pos, 64, False, 500.0, factor, context, low, high, False), torch.float32)


def test_rotary_in_place_with_strides_and_few_or_many_rows():
    for B, H, N in ((1, 8, 5), (32, 8, 1), (2, 3, 20000)):
        for dtype in (torch.bfloat16, torch.float32):
            rows = torch.randn((B, N, 4, H, 64), generator=torch.Generator().manual_seed(N)).to(dtype).cuda()
            before = rows.clone()
            Q, K = (rows[:, :, i].permute(0, 2, 1, 3) for i in range(2))
            pos = torch.arange(N, dtype=torch.float32, device="cuda")
            want = bpt.bpt_rotary(Q, K, pos, rot=32)
            assert torch.equal(rows, before)
            got = bpt.bpt_rotary(Q, K, pos, rot=32, out=(Q, K))
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert torch.equal(rows[:, :, 2:], before[:, :, 2:])      # the values and outputs beside them
            ref, size = reference(before[:, :, 0].permute(0, 2, 1, 3), pos, 32, False, 10000.0, 1.0, 0, 1.0, 32.0, False)
            check(want[0], ref, size, dtype)


def test_rotary_positions_from_the_middle_of_an_array():
    Q = make(2, 2, 13, torch.bfloat16, "heads", 4)
    pos = torch.arange(100, dtype=torch.float32, device="cuda")
    got, _ = bpt.bpt_rotary(Q, None, pos[37:50])
    check(got, *reference(Q, pos[37:50], 64, False, 10000.0, 1.0, 0, 1.0, 32.0, False), torch.bfloat16)


def test_rotary_writes_its_rows_only_and_takes_broadcast_inputs():
    frame = torch.full((2, 3, 12, 72), 7.0, device="cuda")
    out = frame[:, :2, 1:11, 8:]
    one = torch.randn((1, 1, 10, 64), device="cuda")
    x = one.expand(2, 2, 10, 64)          # the same rows for all heads: strides of zero
    pos = torch.arange(20, dtype=torch.float32, device="cuda").view(2, 10)
    bpt.bpt_rotary(x, None, pos, out=(out, None))
    check(out, *reference(x, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, False), torch.float32)
    out.fill_(7.0)
    assert bool((frame == 7.0).all())
    empty = torch.empty((2, 2, 0, 64), device="cuda")
    assert bpt.bpt_rotary(empty, empty, pos[0, :0])[0].shape == empty.shape


def test_rotary_gradient_is_the_transpose():
    # turning is linear: <turn(x), g> = <x, grad>, and the gradient is the reference turned the other way
    Q, K = (make(2, 3, 21, torch.float32, "nodes", s).requires_grad_() for s in (1, 2))
    pos = torch.arange(21, dtype=torch.float32, device="cuda") * 3
    Qr, Kr = bpt.rotary(Q, K, pos, rot=48, interleaved=True)
    g = torch.randn((2, 3, 21, 64), generator=torch.Generator().manual_seed(5)).cuda()
    dQ, dK = torch.autograd.grad((Qr * g).sum() + (Kr * 2 * g).sum(), (Q, K))
    want, size = reference(g, pos, 48, True, 10000.0, 1.0, 0, 1.0, 32.0, True)
    check(dQ, want, size, torch.float32)
    check(dK, 2 * want, 2 * size, torch.float32)
    dQ, = torch.autograd.grad((bpt.rotary(Q, K, pos, rot=48, interleaved=True)[0] * g).sum(), (Q,))   # Kr unused
    check(dQ, want, size, torch.float32)
    Kr_only, = torch.autograd.grad((bpt.rotary(Q, None, pos)[0] * g).sum(), (Q,))
    check(Kr_only, *reference(g, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, True), torch.float32)


def centres(n):
    return np.concatenate([np.arange(n >> l) * float(1 << l) + 0.5 * ((1 << l) - 1) for l in range(n.bit_length())])


@pytest.mark.parametrize("n", [2, 8, 64, 4096])
def test_positions_of_the_nodes_of_a_tree(n):
    g = bpt.bpt_build_graph(n, 2, True)
    assert np.array_equal(bpt.bpt_node_positions(g).cpu().numpy(), centres(n).astype(np.float32))
    g.destroy()


@pytest.mark.parametrize("lengths", [[64, 1, 33], [0, 5, 0, 0, 64, 7, 0], [1], [13] * 40])
@pytest.mark.parametrize("shared", [False, True])
def test_positions_of_the_nodes_of_a_packed_batch(lengths, shared):
    tree = bpt.bpt_build_graph(64, 3, False)
    g = bpt.bpt_build_batch_graph_on(tree, lengths) if shared else bpt.bpt_build_batch_graph(64, 3, False, lengths)
    got = bpt.bpt_node_positions(g).cpu().numpy()
    want = np.full(g.num_nodes, np.nan, dtype=np.float32)
    for level in range(g.num_levels):
        for b in range(g.batch):
            first, count = g.first_row[level, b], g.row_count[level, b]
            want[first:first + count] = np.arange(count) * float(1 << level) + 0.5 * ((1 << level) - 1)
    assert np.array_equal(got, want)
    g.destroy()
    tree.destroy()


def test_rotary_gradients_of_any_layout():
    # as autograd hands them over: rows of [B,N,H,64], different layouts for Q and K, gaps, one value for all
    B, H, N = 2, 3, 37
    pos = torch.arange(N, dtype=torch.float32, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        for of_q, of_k in (("heads", "heads"), ("nodes", "nodes"), ("nodes", "heads"), ("gaps", "gaps")):
            Q, K = (make(B, H, N, dtype, "nodes", s).requires_grad_() for s in (1, 2))
            gq, gk = make(B, H, N, dtype, of_q, 3), make(B, H, N, dtype, of_k, 4)
            got = torch.autograd.grad(bpt.rotary(Q, K, pos), (Q, K), (gq, gk))
            for g, d in zip((gq, gk), got):
                check(d, *reference(g, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, True), dtype)
        Q = make(B, H, N, dtype, "heads", 1).requires_grad_()
        for g in (torch.ones((), dtype=dtype, device="cuda").expand(Q.shape), make(1, 1, N, dtype, "heads", 5).expand(Q.shape),
                  make(B, H, N + 1, dtype, "heads", 6).flatten()[4:4 + Q.numel()].view(Q.shape)):
            d, = torch.autograd.grad(bpt.rotary(Q, None, pos)[0], Q, g)
            check(d, *reference(g, pos, 64, False, 10000.0, 1.0, 0, 1.0, 32.0, True), dtype)


def test_rotary_far_into_memory():
    # rows whose elements lie more than 2^31 apart
    N, H, wide = 1500000, 8, 1600
    rows = torch.empty((1, N, wide), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 31) // wide - 1, (1 << 31) // wide, (1 << 31) // wide + 1, N - 2, N - 1], device="cuda")
    rows[:, at] = torch.randn((1, len(at), wide), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    Q, K = (rows[:, :, 512 * i:512 * (i + 1)].view(1, N, H, 64).permute(0, 2, 1, 3) for i in range(2))
    pos = torch.arange(N, dtype=torch.float32, device="cuda")
    for out in (None, (Q, K)):
        before = [x[:, :, at].clone() for x in (Q, K)]
        for x, y in zip(before, bpt.bpt_rotary(Q, K, pos, out=out)):
            check(y[:, :, at], *reference(x, pos[at], 64, False, 10000.0, 1.0, 0, 1.0, 32.0, False), torch.bfloat16)
