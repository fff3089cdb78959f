"""The operators around a block's linears together, through the example that runs
them: gradients against the formulas in 64 bits, captured graphs against eager calls.

Bounds.  The chain in 64 bits takes the kernels' own codes (a gradient straight through
the rounding has them as constants) and exact values between the operators, the kernels
round to bfloat16: an error of at most 2^-8 of each value that is rounded, of either
sign, so that against a result's root mean square each rounding on the way adds at most
2^-8.  Roundings on the way: of the weight's and the input's gradient two a linear (an
operand, the result), of the GELU's gradient and of the norm's one each, and the kept u
one (the GELU's slope is of order one).
"""
import importlib.util
import os

import pytest
import torch

import paper_2608_03057_amd as T
from conftest import ROOT

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location(
    "feed_forward_half", os.path.join(ROOT, "examples", "feed_forward_half.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)

STEP = 2.0 ** -8


def problem(B=2, S=77, width=144, hidden=320, seed=0, dtype=torch.bfloat16):
    half = example.FeedForwardHalf(width, hidden, dtype)
    gen = torch.Generator().manual_seed(seed + 3)
    x, y, dout, dr = (torch.randn(B, S, width, generator=gen).to("cuda", dtype) for _ in range(4))
    mods = [(0.3 * torch.randn(B, width, generator=gen)).cuda() for _ in range(3)]
    return half, x, y, mods, dout, dr


def masked(W, b):
    return torch.bitwise_and(W.to(torch.int32), -(1 << (8 - b))).double()


def miss(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("b", [8, 5])
@pytest.mark.parametrize("S,width,hidden", [(77, 144, 320), (1, 72, 99), (600, 288, 1152)])
def test_gradients(S, width, hidden, b):
    half, x, y, mods, dout, dr = problem(2, S, width, hidden)
    _, out, kept = half.forward(x, y, mods, b)
    g, up, down = half.backward(dout, dr, kept, y, mods, b)
    r, c1, s1, u, c2, s2 = kept
    C = width
    # The stream and its norm, differentiated by autograd in 64 bits.
    leaves = [t.double().requires_grad_() for t in (x, y, *mods, half.weight)]
    xd, yd, gate, scale, shift, weight = leaves
    rd = xd + gate[:, None] * yd
    d = rd - rd.mean(-1, keepdim=True)
    n = d / (d.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    h = n * weight * (1 + scale[:, None]) + shift[:, None]
    # The linears and the GELU between them, straight through the codes.
    do = dout.double().view(-1, C)
    W1, W2 = (masked(l.W, b) * l.sw.double()[:, None] for l in (half.up, half.down))
    dw2 = do.t() @ (c2.double() * s2.double()[:, None])
    ud = u.double().requires_grad_()
    example.gelu(ud, approximate="tanh").backward(do @ W2)
    dw1 = ud.grad.t() @ (c1.double() * s1.double()[:, None])
    torch.autograd.backward([h, rd], [(ud.grad @ W1).view_as(h), dr.double()])
    assert miss(down[0], dw2) < 2 * STEP
    assert miss(down[1], do.sum(0)) < 1e-5
    # da: 2, du: 3 (u's own rounding is in the reference as well), dw1 and dh: 5.
    assert miss(up[0], dw1) < 5 * STEP
    assert miss(up[1], ud.grad.sum(0)) < 3 * STEP
    # r is rounded before the norm and kept so, and the gradients are once more.
    names = ("dx", "dy", "dgate", "dscale", "dshift", "dweight")
    for name, leaf in zip(names, leaves):
        assert miss(getattr(g, name), leaf.grad) < 7 * STEP, name


def test_training_and_serving_run():
    half, x, y, mods, dout, _ = problem()
    before = [t.clone() for t in (half.up.w, half.down.w, half.weight)]
    loss = half.train_step(x, y, mods, dout, 6, 1.0)
    assert torch.isfinite(loss)
    for old, new in zip(before, (half.up.w, half.down.w, half.weight)):
        assert torch.isfinite(new).all() and not torch.equal(old, new)
    for layer in (half.up, half.down):
        layer.pack()
    r, four = half.serve(x, y, mods)
    r8, out, _ = half.forward(x, y, mods, 8)
    assert torch.equal(r, r8)
    # A 4-bit code is off by at most a quarter of a value (and less than the least
    # step); two operands in each of two linears.
    assert miss(four, out.double()) < 0.5


def everything(half, x, y, mods, dout, dr, b):
    r, out, kept = half.forward(x, y, mods, b)
    g, up, down = half.backward(dout, dr, kept, y, mods, b)
    return [r, out, *(t for t in g if t is not None), *up, *down, *half.serve(x, y, mods)[1:]]


def captured(f):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    return graph, out


def test_captured_steps_of_two_shapes_replayed_in_turn():
    cases = []
    for S, width, hidden in ((77, 144, 320), (530, 288, 600)):
        p = problem(2, S, width, hidden)
        for layer in (p[0].up, p[0].down):
            layer.pack()
        cases.append((p, *captured(lambda p=p: everything(*p, 6))))
    for seed in range(3):
        for p, graph, out in cases:
            new = problem(2, p[1].shape[1], p[1].shape[2], 16, seed=seed + 1)
            for i in (1, 2, 4, 5):
                p[i].copy_(new[i])
            graph.replay()
            eager = everything(*p, 6)
            torch.cuda.synchronize()
            assert all(torch.equal(a, e) for a, e in zip(out, eager))


def test_graphs_that_share_a_workspace():
    """One workspace, two graphs on one stream, each replay after the other's."""
    n = max(T.masked_linear_tokens_backward_workspace_bytes(*s)
            for s in ((1500, 96, 64), (3000, 64, 48)))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    graphs = []
    for M, N, K in ((1500, 96, 64), (3000, 64, 48)):
        g = torch.Generator().manual_seed(M)
        args = [torch.randn(M, N, generator=g).to("cuda", torch.float16),
                torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8).cuda(),
                torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8).cuda(),
                torch.rand(M, generator=g).cuda(), torch.rand(N, generator=g).cuda()]

        def call(args=args):
            return T.masked_linear_tokens_backward(*args, 7, workspace=ws)
        graphs.append((args, *captured(call)))
    for _ in range(3):
        for args, graph, out in graphs:
            for t in out:
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in
                       zip(out, T.masked_linear_tokens_backward(*args, 7)))


def test_on_streams_side_by_side():
    """The same operators on two streams at once, each with its own tensors."""
    problems = [problem(2, 530, 288, 600, seed=s) for s in range(2)]
    for p in problems:
        for layer in (p[0].up, p[0].down):
            layer.pack()
    ref = [everything(*p, 6) for p in problems]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    for _ in range(3):
        outs = []
        for p, s in zip(problems, streams):
            with torch.cuda.stream(s):
                outs.append(everything(*p, 6))
        torch.cuda.synchronize()
        for out, r in zip(outs, ref):
            assert all(torch.equal(a, b) for a, b in zip(out, r))
