"""The 4-bit linear over many tokens, where a workgroup walks several tiles of 256 x 256:
each output type with and without a bias, sums of two steps on, even and odd counts of
128 elements, and M and N that are no whole tiles.

Tolerances: products are exact, the K sums round to fp32 (at most half a step, 2^-24,
each, of the products' magnitudes), the bias is one more sum, the result is rounded once.
"""
import math

import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def values(codes, scales):
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(1).long()
    v = torch.tensor(GRID, dtype=torch.float64, device=DEV)[code & 7]
    v = torch.where(code > 7, -v, v)
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


def operands(M, K, N, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(M, K, generator=g, device=DEV)
    x = x * torch.exp(torch.randn(M, 1, generator=g, device=DEV))
    w = torch.randn(N, K, generator=g, device=DEV) / math.sqrt(K)
    # (A bias of its own for every channel, as large as the sums.)
    bias = torch.arange(N, device=DEV) % 509 / 64.0 - 4.0
    return T.quantize_mx4(x), T.quantize_mx4(w), bias


def check(M, K, N, y_type, bias, seed=0):
    x, w, b = operands(M, K, N, seed)
    y = T.linear_mx4(*x, *w, b if bias else None, out_dtype=y_type)
    xv, wv = values(*x), values(*w)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias:
        ref, size = ref + b.double(), size + b.double().abs()
    sums = (K + 1) * 2.0 ** -24 * size
    tol = HALF[y_type] * (ref.abs() + sums) + sums + TINY[y_type]
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    return x, w, b, y


# Tiles: 10 x 17 (some workgroups have none), 9 x 36 (one or two each), 24 x 24.
SIZES = [(2500, 4104), (2049, 9008), (6000, 6136)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("K", [300, 512, 640, 1152])        # 3, 4, 5 and 9 of 128
@pytest.mark.parametrize("y_type", list(HALF))
@pytest.mark.parametrize("bias", [True, False])
def test_walk(M, N, K, y_type, bias):
    check(M, K, N, y_type, bias, seed=M + K)


@pytest.mark.parametrize("y_type", list(HALF))
def test_walk_of_tokens_alone(y_type):
    """The walk's rows as those of the same tokens a few at a time."""
    x, w, b, y = check(2500, 640, 4104, y_type, True, seed=1)
    for first in (0, 255, 256, 1000, 2468):
        few = T.linear_mx4(x[0][first:first + 32], x[1][first:first + 32], *w, b,
                           out_dtype=torch.float32)
        size = values(x[0][first:first + 32], x[1][first:first + 32]).abs() @ \
            values(*w).abs().t() + b.double().abs()
        sums = 2 * 641 * 2.0 ** -24 * size
        off = (y[first:first + 32].double() - few.double()).abs()
        assert bool((off <= HALF[y_type] * (few.double().abs() + sums) + sums +
                     TINY[y_type]).all())


@pytest.mark.parametrize("y_type", list(HALF))
@pytest.mark.parametrize("K", [300, 1152])
def test_walk_writes_its_output_only(K, y_type):
    M, N = 2049, 9008
    x, w, b, y = check(M, K, N, y_type, True, seed=2)
    flat = torch.full((M * N + 2048,), 7.0, dtype=y_type, device=DEV)
    got = T.linear_mx4(*x, *w, b, y=flat[1024:1024 + M * N].view(M, N))
    assert torch.equal(got, y)
    assert bool((flat[:1024] == 7).all()) and bool((flat[1024 + M * N:] == 7).all())


def test_walk_of_scales_that_are_not_numbers():
    """A block without a number reaches its token's row or its channel's column only,
    also across an odd count of 128 elements, where a request of scales reaches into the
    next row's."""
    for K in (300, 640):
        x, w, b, y = check(2500, K, 4104, torch.bfloat16, True, seed=3)
        sx, sw = x[1].clone(), w[1].clone()
        sx[700, 0], sx[256, -1], sw[513, 0] = 255, 255, 255
        got = T.linear_mx4(x[0], sx, w[0], sw, b)
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[700], bad[256], bad[:, 513] = True, True, True
        assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], y[~bad])


def test_walk_captured_and_replayed():
    x, w, b, _ = check(2500, 640, 4104, torch.bfloat16, True, seed=4)

    def f():
        return T.linear_mx4(*x, *w, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = f()
    for seed in range(3):
        new = operands(2500, 640, 4104, seed + 5)[0]
        x[0].copy_(new[0])
        x[1].copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, f())


@pytest.mark.parametrize("M,N", [(100, 70), (2500, 1290), (2500, 9008)])
@pytest.mark.parametrize("y_type", list(HALF))
def test_no_channels_over_many_tokens(M, N, y_type):
    """Sums of nothing in tiles of 64, 128 and 256: the bias, or zeros."""
    x, w = (T.quantize_mx4(torch.zeros(n, 0, device=DEV)) for n in (M, N))
    bias = operands(1, 32, N, 0)[2]
    y = T.linear_mx4(*x, *w, bias, out_dtype=y_type)
    assert torch.equal(y, bias.to(y_type).expand(M, N))
    assert not T.linear_mx4(*x, *w, out_dtype=y_type).any()
