"""The feed-forward half of a quantized transformer block: trained on low-bit codes,
and served in four bits.

The attention half's output enters the residual stream through its gate, the stream is
normed and modulated, and two linears with a GELU between them give the half's output.
In training every linear takes int8 codes with one scale per token, and those codes are
all that is kept of its input for the backward pass; the weights that are trained are
fp32 and quantized again after each step.  In serving both linears take 4-bit
microscaled codes of activations and weights.

    python examples/feed_forward_half.py --batch 2 --tokens 1024 --steps 5
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_03057_amd as T  # noqa: E402

gelu = torch.nn.functional.gelu


class Linear:
    """A trained fp32 weight [N, K] and bias; its 8-bit codes with one scale per
    channel, and its 4-bit ones."""

    def __init__(self, N, K, gen, device):
        self.w = (torch.randn(N, K, generator=gen) / math.sqrt(K)).to(device)
        self.bias = (0.02 * torch.randn(N, generator=gen)).to(device)
        self.quantize()

    def quantize(self):
        self.W, self.sw = T.quantize_tokens(self.w)     # (a scale a row, as tokens have)

    def pack(self):
        """The 4-bit codes, once before serving."""
        self.packed = T.quantize_mx4(self.w)

    def __call__(self, codes, scales, b, dtype):
        return T.masked_linear_tokens(codes, self.W, scales, self.sw, b, self.bias,
                                      out_dtype=dtype)

    def backward(self, dy, codes, scales, b):
        """Gradients of the input, the weight and the bias."""
        return T.masked_linear_tokens_backward(dy, codes, self.W, scales, self.sw, b)

    def serve(self, x, dtype):
        return T.linear_mx4(*T.quantize_mx4(x), *self.packed, self.bias, out_dtype=dtype)


class FeedForwardHalf:
    def __init__(self, width, hidden, dtype=torch.bfloat16, device="cuda", seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype = dtype
        self.up = Linear(hidden, width, gen, device)
        self.down = Linear(width, hidden, gen, device)
        self.weight = (1 + 0.1 * torch.randn(width, generator=gen)).to(device)

    def forward(self, x, y, mods, b):
        """(r, out, what the backward pass takes): the stream x [B, S, C] with the branch
        y, and the half's output, which a gate of its own takes into r; mods are the
        branch's gate, the scale and the shift, fp32 [B, C]."""
        B, S, C = x.shape
        gate, scale, shift = mods
        r, h = T.residual_norm(x, y, gate, weight=self.weight, scale=scale, shift=shift)
        c1, s1 = T.quantize_tokens(h.view(B * S, C))
        u = self.up(c1, s1, b, self.dtype)
        c2, s2 = T.quantize_tokens(gelu(u, approximate="tanh"))
        return r, self.down(c2, s2, b, self.dtype).view(B, S, C), (r, c1, s1, u, c2, s2)

    def backward(self, dout, dr, kept, y, mods, b):
        """Gradients from those of the half's output and of r: of x, y, the
        modulations and the norm's weight (ResidualGrads), and (dw, dbias) of both
        linears."""
        r, c1, s1, u, c2, s2 = kept
        B, S, C = r.shape
        gate, scale, shift = mods
        da, *down = self.down.backward(dout.view(B * S, C), c2, s2, b)
        du = torch.ops.aten.gelu_backward(da, u, approximate="tanh")
        dh, *up = self.up.backward(du, c1, s1, b)
        g = T.residual_norm_backward(dh.view(B, S, C), dr, r, y, gate, weight=self.weight,
                                     scale=scale, shift=shift)
        return g, up, down

    def train_step(self, x, y, mods, target, b, rate):
        """One gradient step on mean (out - target)^2; returns the loss before it."""
        _, out, kept = self.forward(x, y, mods, b)
        miss = out.float() - target.float()
        # (The factor 2 / n comes last, where it leaves half's range.)
        g, up, down = self.backward(miss.to(self.dtype), None, kept, y, mods, b)
        f = 2 * rate / miss.numel()
        for layer, (dw, dbias) in ((self.up, up), (self.down, down)):
            layer.w.add_(dw, alpha=-f)
            layer.bias.add_(dbias, alpha=-f)
            layer.quantize()
        self.weight.add_(g.dweight, alpha=-f)
        return miss.square().mean()

    def serve(self, x, y, mods):
        """(r, out) with both linears in four bits."""
        B, S, C = x.shape
        gate, scale, shift = mods
        r, h = T.residual_norm(x, y, gate, weight=self.weight, scale=scale, shift=shift)
        a = gelu(self.up.serve(h.view(B * S, C), self.dtype), approximate="tanh")
        return r, self.down.serve(a, self.dtype).view(B, S, C)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batch", type=int, default=2)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--width", type=int, default=1152)
    p.add_argument("--hidden", type=int, default=4608)
    p.add_argument("--bits", type=int, default=6)
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--rate", type=float, default=2.0)
    a = p.parse_args()
    half = FeedForwardHalf(a.width, a.hidden)
    gen = torch.Generator().manual_seed(1)
    x, y, target = (torch.randn(a.batch, a.tokens, a.width, generator=gen).to("cuda", torch.bfloat16)
                    for _ in range(3))
    mods = [0.3 * torch.randn(a.batch, a.width, generator=gen).cuda() for _ in range(3)]
    for i in range(a.steps):
        loss = half.train_step(x, y, mods, 0.1 * target, a.bits, a.rate)
        print(f"step {i}: loss {loss:.4e}")
    for layer in (half.up, half.down):
        layer.pack()
    _, out, _ = half.forward(x, y, mods, 8)
    _, four = half.serve(x, y, mods)
    miss = (four.float() - out.float()).square().mean().sqrt() / out.float().square().mean().sqrt()
    print(f"four bits against eight: {miss:.3f} of the output")


if __name__ == "__main__":
    main()
