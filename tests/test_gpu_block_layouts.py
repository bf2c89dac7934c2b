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
