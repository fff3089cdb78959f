"""The block's operators together, through the example that runs them: a step
of the attention half against the same half in 64 bits, its captured graph
against the eager step, a calibration step's gradients against the formulas.

Bounds.  The two sides round to bfloat16 (relative 2^-9) at the same places but
after sums in another precision, so their values differ by single roundings:
through scores of a few units that is about 3 * 2^-8 of an attention's
output.  Where they are quantized again, a difference e moves a code, that is
by the scale s, with probability e / s: root mean square sqrt(s e), with
s = 4 / 127 and e = 2^-8 of the activations 1.1%.  Four such linears and two
attentions: 3%; asserted is 4% of the root mean square of what the half adds
to its input.  (A head, key, mask or rotation mixed up gives more than 50%.)
"""
import importlib.util
import os

import pytest
import torch

import paper_2608_03057_amd as T
from conftest import ROOT

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location(
    "attention_half", os.path.join(ROOT, "examples", "attention_half.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def problem(B=2, side=12, width=288, heads=4, words=77, text_width=160, dtype=torch.bfloat16):
    block = example.AttentionHalf(width, heads, side, text_width, dtype)
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(B, side * side, width, generator=gen).to("cuda", dtype)
    text = torch.randn(B, words, text_width, generator=gen).to("cuda", dtype)
    lengths = torch.tensor([words, 9][:B], dtype=torch.int32, device="cuda")
    return block, x, text, lengths


class Plain:
    """The half in 64 bits on the CPU, rounded where the framework's tensors are."""

    def __init__(self, block):
        self.o = block

    def round(self, t):
        return t.to(self.o.dtype).double()

    def linear(self, layer, x, b):
        s = (x.abs().amax(-1, keepdim=True).float() * torch.tensor(1 / 127)).double()
        codes = torch.round(torch.where(s > 0, x / s, torch.zeros_like(x))).clamp(-127, 127)
        keep = (0xff << (8 - b)) & 0xff
        W = (layer.W.cpu().to(torch.int16) & (keep - 256 if keep > 127 else keep)).double()
        return self.round(codes @ W.T * s * layer.sw.cpu().double() + layer.bias.cpu().double())

    def normed(self, x, w):
        cos, sin = (t.cpu().double()[None, :, None] for t in self.o.rope[:2])
        n = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.cpu().double()
        half = cos.shape[-1]
        a, c = n[..., :half], n[..., half:2 * half]
        return self.round(torch.cat([a * cos - c * sin, a * sin + c * cos, n[..., 2 * half:]], -1))

    def attention(self, q, k, v, lengths=None):
        z = torch.einsum("bihd,bjhd->bhij", q, k) * q.shape[-1] ** -0.5
        if lengths is not None:
            j = torch.arange(k.shape[1])
            z = z.masked_fill(j[None, None, None] >= lengths.cpu()[:, None, None, None],
                              float("-inf"))
        return self.round(torch.einsum("bhij,bjhd->bihd", z.softmax(-1), v)), z

    def step(self, x, text, lengths, b):
        o, x, text = self.o, x.cpu().double(), text.cpu().double()
        B, S, C = x.shape
        shape = (B, S, o.heads, o.dim)
        kv = self.linear(o.kv_cross, text, b).view(B, -1, 2, o.heads, o.dim)
        q, k, v = self.linear(o.qkv, x, b).view(B, S, 3, o.heads, o.dim).unbind(2)
        a, _ = self.attention(self.normed(q, o.wq), self.normed(k, o.wk), v)
        x = self.round(x + self.linear(o.out, a.reshape(B, S, C), b))
        q = self.linear(o.q_cross, x, b).view(shape)
        a, _ = self.attention(q, kv[:, :, 0], kv[:, :, 1], lengths)
        return self.round(x + self.linear(o.out_cross, a.reshape(B, S, C), b))


@pytest.mark.parametrize("b", [8, 5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_step_against_the_plain_half(b, dtype):
    block, x, text, lengths = problem(dtype=dtype)
    y = block.step(x, block.prompt(text, b), lengths, b).cpu().double()
    want = Plain(block).step(x, text, lengths, b)
    added = want - x.cpu().double()
    assert float((y - want).norm() / added.norm()) < 0.04


def test_graph_replays_the_eager_step():
    block, x, text, lengths = problem()
    kv = block.prompt(text, 6)
    graph, y = example.capture(lambda: block.step(x, kv, lengths, 6))
    for r in range(4):
        x.copy_(torch.roll(x, 1, 1))
        lengths.copy_(torch.roll(lengths, 1))
        want = block.step(x, kv, lengths, 6)
        y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), r


def test_calibration_gradients_and_descent():
    """The norms' gradients against differentiating the plain half in 64 bits:
    sums over 1152 heads of terms rounded to bfloat16 in between (relative
    2^-8 each, partly cancelling): 5% of the gradient's norm."""
    block, x, _, _ = problem()
    q, k, v = block.heads_of(x, 8)
    target, _ = T.attention(*block.normed(q, k), v)
    q, k, v = (t.cpu().double() for t in block.heads_of(x, 4))
    plain = Plain(block)
    plain.round = lambda t: t
    wq, wk = (t.cpu().double().requires_grad_() for t in (block.wq, block.wk))
    a, _ = plain.attention(plain.normed(q, wq), plain.normed(k, wk), v)
    loss = (a - target.cpu().double()).square().mean()
    loss.backward()
    loss = float(loss.detach())
    got, dwq, dwk = block.calibrate_step(x, 4, target, rate=0.0)
    assert abs(float(got) / loss - 1) < 0.02
    for g, w in ((dwq, wq), (dwk, wk)):
        assert float((g.cpu().double() - w.grad).norm() / w.grad.norm()) < 0.05
    # A step along the gradient brings the loss down by about rate |gradient|^2.
    rate = 0.05 * loss / float(sum(w.grad.square().sum() for w in (wq, wk)))
    first, _, _ = block.calibrate_step(x, 4, target, rate)
    second, _, _ = block.calibrate_step(x, 4, target, 0.0)
    assert float(second) < float(first)
