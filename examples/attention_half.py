"""The attention half of a quantized transformer block, run as a sampler runs it.

Every linear takes int8 codes with one scale per token and the shared 8-bit
weight at the bits of the denoising stage; between them stand the norm and
rotation of the heads of q and k, attention of the image tokens among
themselves, and their attention over the prompt's words, whose keys and values
are computed once for all steps.  The launches of a step are captured in a
HIP graph and replayed.

With --calibrate the weights of the head norms are fitted afterwards: gradient
steps that bring the attention of the low-bit projections towards that of the
8-bit ones.

    python examples/attention_half.py --batch 2 --side 64 --words 300
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_03057_amd as T  # noqa: E402


def rope_tables(side, rot, device):
    """(cos, sin) [side * side, rot / 2] of an image's tokens: the first half of
    the frequencies turns with the row, the second with the column."""
    half = rot // 2
    rows = half // 2
    i = torch.arange(half, dtype=torch.float64)
    freq = 100.0 ** -(torch.where(i < rows, i, i - rows) / max(rows, 1))
    at = torch.arange(side * side)
    place = torch.where(i[None] < rows, (at // side)[:, None], (at % side)[:, None])
    angle = place * freq
    return angle.cos().float().to(device), angle.sin().float().to(device)


class Linear:
    """An 8-bit weight [N, K] with one scale per channel, and a bias."""

    def __init__(self, N, K, gen, device):
        W = torch.randn(N, K, generator=gen) / math.sqrt(K)
        self.sw = (W.abs().amax(1) / 127).to(device)
        self.W = torch.round(W / (W.abs().amax(1, keepdim=True) / 127)).to(torch.int8).to(device)
        self.bias = (0.02 * torch.randn(N, generator=gen)).to(device)

    def __call__(self, codes, scales, b, dtype):
        return T.masked_linear_tokens(codes, self.W, scales, self.sw, b, self.bias,
                                      out_dtype=dtype)


class AttentionHalf:
    def __init__(self, width, heads, side, text_width, dtype=torch.bfloat16, device="cuda",
                 seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.width, self.heads, self.dim, self.dtype = width, heads, width // heads, dtype
        self.qkv = Linear(3 * width, width, gen, device)
        self.out = Linear(width, width, gen, device)
        self.q_cross = Linear(width, width, gen, device)
        self.kv_cross = Linear(2 * width, text_width, gen, device)
        self.out_cross = Linear(width, width, gen, device)
        self.wq, self.wk = ((1 + 0.1 * torch.randn(self.dim, generator=gen)).to(device)
                            for _ in range(2))
        self.rope = (*rope_tables(side, self.dim // 4 * 4, device), None)

    def prompt(self, text, b):
        """Keys and values [B, words, 2, heads, dim] of the prompt's states."""
        B, S, C = text.shape
        kv = self.kv_cross(*T.quantize_tokens(text.view(B * S, C)), b, self.dtype)
        return kv.view(B, S, 2, self.heads, self.dim)

    def heads_of(self, x, b):
        """q, k and v [B, S, heads, dim] of tokens x, slices of one projection."""
        B, S, C = x.shape
        qkv = self.qkv(*T.quantize_tokens(x.view(B * S, C)), b, self.dtype)
        return qkv.view(B, S, 3, self.heads, self.dim).unbind(2)

    def normed(self, q, k):
        return T.qk_norm_rotate(q, k, self.wq, self.wk, self.rope, self.rope)

    def step(self, x, kv, lengths, b):
        """The block's attention half at b bits: x [B, S, width], the prompt's kv,
        its number of words int32 [B]."""
        B, S, C = x.shape
        q, k, v = self.heads_of(x, b)
        q, k = self.normed(q, k)
        a, _ = T.attention(q, k, v)
        x = x + self.out(*T.quantize_tokens(a.view(B * S, C)), b, self.dtype).view(B, S, C)
        q = self.q_cross(*T.quantize_tokens(x.view(B * S, C)), b, self.dtype)
        a, _ = T.attention(q.view(B, S, self.heads, self.dim), kv[:, :, 0], kv[:, :, 1],
                           kv_lengths=lengths)
        return x + self.out_cross(*T.quantize_tokens(a.view(B * S, C)), b,
                                  self.dtype).view(B, S, C)

    def calibrate_step(self, x, b, target, rate):
        """One gradient step of the norms' weights on mean (a - target)^2, a the
        attention of x at b bits; returns the loss before it and the gradients."""
        q, k, v = self.heads_of(x, b)
        qn, kn = self.normed(q, k)
        a, lse = T.attention(qn, kn, v, want_lse=True)
        miss = a.float() - target.float()
        # The factor 2 / n comes last: with it, half's range would not hold this.
        da = miss.to(self.dtype)
        dq, dk, _ = T.attention_backward(da, qn, kn, v, a, lse)
        _, _, dwq, dwk = T.qk_norm_rotate_backward(dq, dk, q, k, self.wq, self.wk, self.rope,
                                                   self.rope)
        f = 2 / miss.numel()
        self.wq -= rate * f * dwq
        self.wk -= rate * f * dwk
        return miss.square().mean(), f * dwq, f * dwk


def capture(f):
    """f's launches as a graph, and the tensor that each replay writes."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()                     # kernels loaded
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = f()
    return graph, y


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batch", type=int, default=2)
    p.add_argument("--side", type=int, default=64, help="image tokens a side")
    p.add_argument("--width", type=int, default=1152)
    p.add_argument("--heads", type=int, default=16)
    p.add_argument("--words", type=int, default=300)
    p.add_argument("--text-width", type=int, default=4096)
    p.add_argument("--bits", type=int, nargs="+", default=[8, 6, 5, 4], help="of each stage")
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--calibrate", type=int, default=0, metavar="STEPS")
    a = p.parse_args()
    block = AttentionHalf(a.width, a.heads, a.side, a.text_width)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(a.batch, a.side ** 2, a.width, generator=gen).to("cuda", torch.bfloat16)
    text = torch.randn(a.batch, a.words, a.text_width, generator=gen).to("cuda", torch.bfloat16)
    lengths = torch.randint(1, a.words + 1, (a.batch,), generator=gen).int().cuda()
    for stage, b in enumerate(a.bits):
        kv = block.prompt(text, b)
        graph, y = capture(lambda: block.step(x, kv, lengths, b))
        graph.replay()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(a.steps):
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        print(f"stage {stage}: {b} bits, {start.elapsed_time(end) / a.steps * 1e3:.1f} us a step, "
              f"rms {y.float().square().mean().sqrt():.4f}")
    if a.calibrate:
        b = a.bits[-1]
        q, k, v = block.heads_of(x, 8)
        target, _ = T.attention(*block.normed(q, k), v)
        for i in range(a.calibrate):
            loss, _, _ = block.calibrate_step(x, b, target, rate=1e3)
            print(f"calibration step {i}: loss {loss:.3e}")


if __name__ == "__main__":
    main()
