"""The operators of a gated block as they are used together, around graph self-attention: a pre-norm block with rotary positions
on the graph of one tree and on the graph of a packed batch, forward and backward through torch, against 64 bits.

Tolerance.  On the way from the inputs to the output nine tensors are rounded to bf16 (h, Q | K | V, turned Q and K, the attention's
output, its projection, the stream, h again, the hidden activations, the block's output): at most 2^-8 of each one's 2-norm, and the
maps between them have norms near 1 with these parameters, so that the result is off by at most 9 * 2^-8 of its 2-norm, and a
gradient, whose way back rounds as many tensors again and meets those of the way out, by 18 * 2^-8.
"""
import pytest
import torch

from paper_1911_04070_amd import binding as bpt

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8
HEADS, D, F = 2, 128, 264


def parameters(seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    p = {w: (r(D, D) * D ** -0.5).bfloat16() for w in ("Wq", "Wk", "Wv", "Wo")}
    p.update(Wg=(r(D, F) * D ** -0.5).bfloat16(), Wu=(r(D, F) * D ** -0.5).bfloat16(), Wd=(r(F, D) * F ** -0.5).bfloat16(),
             gate=(0.5 + 0.1 * r(1, D)).bfloat16())
    for name in ("n1", "n2", "n3", "n4"):
        p[name] = 1 + 0.1 * r(D)
    return {k: v.cuda().requires_grad_() for k, v in p.items()}


def block(g, x, p, rel, pos):
    N = g.num_nodes
    _, h = bpt.residual_norm(x, None, pre="rms", pre_gain=p["n1"])
    q, k, v = ((h @ p[w]).view(1, N, HEADS, 64).permute(0, 2, 1, 3) for w in ("Wq", "Wk", "Wv"))
    q, k = bpt.rotary(q, k, pos, rot=32)
    o = bpt.graph_attention(g, q, k, v, rel, scale=0.125).permute(0, 2, 1, 3).reshape(N, D)
    x, h = bpt.residual_norm(x, o @ p["Wo"], p["gate"], post="rms", pre="rms", post_gain=p["n2"], pre_gain=p["n3"], gate_rows=N)
    x, h = bpt.residual_norm(x, bpt.gated_ffn(h, p["Wg"], p["Wu"], p["Wd"]), pre="layer", pre_gain=p["n4"], residual_scale=0.5)
    return x, h


def plain(g, x, p, rel, pos):
    N = g.num_nodes
    rms = lambda v, gain: v / ((v * v).mean(1, keepdim=True) + 1e-5).sqrt() * gain
    h = rms(x, p["n1"])
    w = pos.double()[:, None] * 10000.0 ** (-torch.arange(16, dtype=torch.float64, device="cuda") / 16)

    def turn(t):   # [H, N, 64]
        a, b = t[..., :16], t[..., 16:32]
        return torch.cat([a * w.cos() - b * w.sin(), b * w.cos() + a * w.sin(), t[..., 32:]], -1)

    q, k, v = ((h @ p[m]).view(N, HEADS, 64).transpose(0, 1) for m in ("Wq", "Wk", "Wv"))
    q, k = turn(q), turn(k)
    row_ptr, col, ids = (torch.from_numpy(a).long().cuda() for a in g.csr_to_host())
    row = torch.repeat_interleave(torch.arange(N, device="cuda"), row_ptr[1:] - row_ptr[:-1])
    s = 0.125 * (q[:, row] * (k[:, col] + rel.reshape(-1, 64)[ids])).sum(-1)
    e = torch.exp(s - s.max())
    weight = e / torch.zeros((HEADS, N), dtype=torch.float64, device="cuda").index_add(1, row, e)[:, row]
    o = torch.zeros((HEADS, N, 64), dtype=torch.float64, device="cuda").index_add(1, row, weight[..., None] * v[:, col])
    x = x + p["gate"] * rms(o.transpose(0, 1).reshape(N, D) @ p["Wo"], p["n2"])
    h = rms(x, p["n3"])
    u = h @ p["Wg"]
    x = 0.5 * x + ((u * torch.sigmoid(u)) * (h @ p["Wu"])) @ p["Wd"]
    c = x - x.mean(1, keepdim=True)
    return x, c / ((c * c).mean(1, keepdim=True) + 1e-5).sqrt() * p["n4"]


@pytest.mark.parametrize("lengths", [None, [64, 5, 33, 1]])
def test_block(lengths):
    print("block", lengths, flush=True)
    g = bpt.bpt_build_graph(64, 2, True) if lengths is None else bpt.bpt_build_batch_graph(64, 2, True, lengths)
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((g.num_nodes, D), generator=gen).bfloat16().cuda().requires_grad_()
    rel = (0.02 * torch.randn((g.num_levels, g.rel_width, 64), generator=gen)).bfloat16().cuda()
    dy, dh = (torch.randn((g.num_nodes, D), generator=gen).bfloat16().cuda() for _ in range(2))
    p = parameters(4)
    pos = bpt.bpt_node_positions(g)
    y, h = block(g, x, p, rel, pos)
    grads = torch.autograd.grad((y, h), [x, *p.values()], (dy, dh))
    x64 = x.detach().double().requires_grad_()
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    y64, h64 = plain(g, x64, p64, rel.double(), pos)
    want = torch.autograd.grad((y64, h64), [x64, *p64.values()], (dy.double(), dh.double()))
    off = lambda a, b: float((a.detach().double() - b.detach()).norm() / b.detach().norm())
    assert off(y, y64) <= 9 * STEP and off(h, h64) <= 9 * STEP
    for name, a, b in zip(["x", *p], grads, want):
        assert a.shape == b.shape and off(a, b) <= 18 * STEP, (name, off(a, b))
    g.destroy()


def test_block_captured_while_an_eager_graph_of_it_lives():
    # forward and backward captured into a HIP graph; the eager graph of other leaves stays alive, and every replay is compared
    g = bpt.bpt_build_graph(64, 2, True)
    gen = torch.Generator().manual_seed(5)
    x0 = torch.randn((g.num_nodes, D), generator=gen).bfloat16().cuda()
    rel = (0.02 * torch.randn((g.num_levels, g.rel_width, 64), generator=gen)).bfloat16().cuda()
    dy = torch.randn((g.num_nodes, D), generator=gen).bfloat16().cuda()
    pos = bpt.bpt_node_positions(g)

    def parts(x, p):       # the operators of this library alone: no library products in the captured graph
        _, h = bpt.residual_norm(x, None, pre="rms", pre_gain=p["n1"])
        q = h.view(1, -1, HEADS, 64).permute(0, 2, 1, 3)
        q, k = bpt.rotary(q, q, pos)
        o = bpt.graph_attention(g, q, k, k, rel, scale=0.125).permute(0, 2, 1, 3).reshape(-1, D)
        x, h = bpt.residual_norm(x, o, p["gate"], post="rms", pre="rms", post_gain=p["n2"], pre_gain=p["n3"], gate_rows=g.num_nodes)
        return bpt.residual_norm(x, bpt.gated_ffn(h, p["Wg"], p["Wu"], p["Wd"]), pre="layer", pre_gain=p["n4"])

    names = ("n1", "n2", "n3", "n4", "gate", "Wg", "Wu", "Wd")

    def step(x, p):
        y, h = parts(x, p)
        return (y.detach(), h.detach()) + torch.autograd.grad((y, h), [x] + [p[k] for k in names], (dy, dy))

    x, p = x0.clone().requires_grad_(), parameters(6)
    alive = parts(x, p)
    want = step(x, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        xs, ps = x0.clone().requires_grad_(), {k: v.detach().clone().requires_grad_() for k, v in p.items()}
        step(xs, ps)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = step(xs, ps)
    torch.cuda.synchronize()
    for _ in range(3):
        for v in got:
            v.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(step(x, p), want))
    assert all(torch.equal(a, b) for a, b in zip(alive, want[:2]))
    del graph, got
    g.destroy()


def test_two_streams_at_once():
    # the same calls on two streams, each with its own buffers, nothing waited for in between
    gen = torch.Generator().manual_seed(7)
    inputs = [torch.randn((3000, D), generator=gen).bfloat16().cuda() for _ in range(2)]
    p = {k: v.detach() for k, v in parameters(8).items()}

    def work(x):
        y, h, stats = bpt.bpt_residual_norm_fwd(x, x, p["gate"], post="rms", pre="layer", post_gain=p["n1"], gate_rows=3000, want_stats=True)
        Y = bpt.bpt_gated_ffn_fwd(h, p["Wg"], p["Wu"], p["Wd"])
        return (Y,) + bpt.bpt_gated_ffn_bwd(h, p["Wg"], p["Wu"], p["Wd"], Y) + tuple(
            bpt.bpt_residual_norm_bwd(x, x, p["gate"], stats, y, Y, post="rms", pre="layer", post_gain=p["n1"], gate_rows=3000).values())

    want = [work(x) for x in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for x, s in zip(inputs, streams):
            with torch.cuda.stream(s):
                got.append(work(x))
    torch.cuda.synchronize()
    for i, v in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(v, want[i % 2]))


def test_gradients_off_the_boundary():
    # autograd may hand over a gradient that starts anywhere
    x = torch.randn((5, D), generator=torch.Generator().manual_seed(9)).bfloat16().cuda().requires_grad_()
    p = parameters(10)
    dy = torch.randn((5, D), generator=torch.Generator().manual_seed(11)).bfloat16().cuda()
    off = torch.zeros(5 * D + 1, dtype=torch.bfloat16, device="cuda")[1:].view(5, D).copy_(dy)
    for f in (lambda: bpt.residual_norm(x, x, pre="none")[0], lambda: bpt.residual_norm(x, x, pre="rms")[1],
              lambda: bpt.gated_ffn(x, p["Wg"], p["Wu"], p["Wd"])):
        assert torch.equal(*(torch.autograd.grad(f(), x, g)[0] for g in (dy, off)))
