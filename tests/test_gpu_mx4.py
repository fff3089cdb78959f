"""4-bit microscaled codes and the linear on them.

Codes are decisions on exact quotients, so they are compared bit by bit with those
of the definition in 64 bits.  The linear's products are exact; its K sums round to
fp32 (half a step, 2^-24, of what is at most the sum of the products' magnitudes,
each), then the bias is added and the result is rounded to its type.
"""
import math

import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def definition(x):
    """(codes [M, K'/2], scales [M, K'/32]) of x [M, K], in 64 bits."""
    M, K = x.shape
    wide = torch.zeros(M, (K + 127) // 128 * 128, dtype=torch.float64, device=x.device)
    wide[:, :K] = x.double()
    b = wide.view(M, -1, 32)
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    e = torch.frexp(torch.where(bad, torch.ones_like(top), top))[1] - 1 - 2
    e = torch.where(top == 0, torch.full_like(e, -127), e).clamp(min=-127)
    a = b / torch.exp2(e.double())[..., None]
    place = torch.zeros_like(b, dtype=torch.int32)
    for i in range(7):
        middle = (GRID[i] + GRID[i + 1]) / 2
        place += ((a.abs() >= middle) if i % 2 else (a.abs() > middle)).int()
    code = place + 8 * torch.signbit(a).int()
    code[bad] = 0
    code = code.view(M, -1)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8), scales.to(torch.uint8)


def values(codes, scales):
    """What they stand for, in 64 bits, [rows, K']."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(1).long()
    v = torch.tensor(GRID, dtype=torch.float64, device=codes.device)[code & 7]
    v = torch.where(code > 7, -v, v)
    s = torch.where(scales == 255, torch.nan, torch.exp2(scales.double() - 127))
    return v * s.repeat_interleave(32, 1)


def unsigned_zeros(codes):
    """Codes one by one, a zero of either sign as zero."""
    each = torch.stack((codes & 15, codes >> 4), -1)
    return torch.where(each == 8, 0, each)


def check_codes(x):
    codes, scales = T.quantize_mx4(x)
    rc, rs = definition(x)
    assert torch.equal(scales, rs)
    assert torch.equal(unsigned_zeros(codes), unsigned_zeros(rc))
    return codes, scales


def normal(*shape, dtype=torch.float32, seed=0, f=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * f).to(dtype)


@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("M,K", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 127), (4, 128), (7, 129),
                                 (3, 640), (2, 1152), (9, 1153), (1, 4608), (300, 77), (2, 131071)])
def test_codes(M, K, dtype):
    spread = torch.exp(2 * normal(M, 1, seed=K))
    check_codes((normal(M, K, seed=M) * spread).to(dtype))


@pytest.mark.parametrize("dtype", list(HALF))
def test_every_place_of_the_grid(dtype):
    """Every quotient of an eighth to 8, the middles between codes among them, in
    blocks of every exponent of the type."""
    lo, hi = {torch.float32: (-126, 127), torch.bfloat16: (-126, 127),
              torch.float16: (-14, 15)}[dtype]
    q = torch.arange(-63, 64, device=DEV) / 8.0
    q = q[q.abs() <= 7.875]
    rows = []
    for e in range(lo + 2, hi - 1):
        block = torch.full((len(q), 32), 4.0, device=DEV, dtype=torch.float64)
        block[:, 3], block[:, 31] = q, -q
        rows.append(block * 2.0 ** e)
    x = torch.cat(rows).to(dtype)
    assert torch.isfinite(x).all()
    check_codes(x)


def test_subnormals_and_zeros():
    x = torch.zeros(6, 128, device=DEV)
    x[1, 3] = 2.0 ** -149
    x[2] = 2.0 ** -127 * torch.linspace(-1, 1, 128, device=DEV)
    x[3, :32] = 2.0 ** -125 * torch.linspace(0, 1.99, 32, device=DEV)
    x[4, 40] = -0.0
    x[5, 99] = 3.4028234663852886e38
    check_codes(x)
    check_codes(x.bfloat16())
    check_codes((x * 2.0 ** 115).half())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", list(HALF))
def test_not_finite(bad, dtype):
    x = normal(4, 200, dtype=dtype)
    x[1, 40], x[3, 199] = bad, bad
    codes, scales = check_codes(x)
    want = torch.zeros(4, 8, dtype=torch.bool, device=DEV)
    want[1, 1] = want[3, 6] = True
    assert torch.equal(scales == 255, want)
    w, sw = T.quantize_mx4(normal(70, 200, seed=2))
    for M in (4, 128):
        y = T.linear_mx4(codes.repeat(M // 4, 1), scales.repeat(M // 4, 1), w, sw)
        rows = torch.isnan(y).all(1)
        assert rows.tolist() == [False, True, False, True] * (M // 4)
        assert torch.isfinite(y[~rows]).all()


def test_strided_rows_and_given_outputs():
    wide = normal(9, 3, 200, dtype=torch.bfloat16)
    for x in (wide[:, 1], wide[:, 2, 3:150], wide[::2, 0, 1:]):
        codes, scales = check_codes(x)
        out, s = torch.full_like(codes, 9), torch.full_like(scales, 9)
        got = T.quantize_mx4(x, out, s)
        assert got[0] is out and got[1] is s and torch.equal(out, codes) and torch.equal(s, scales)


@pytest.mark.parametrize("M,K", [(0, 64), (5, 0)])
def test_no_codes(M, K):
    codes, scales = T.quantize_mx4(torch.zeros(M, K, device=DEV))
    assert codes.shape == (M, (K + 127) // 128 * 64) and scales.shape == (M, (K + 127) // 128 * 4)
    w, sw = T.quantize_mx4(torch.ones(6, K, device=DEV))
    bias = normal(6)
    y = T.linear_mx4(codes, scales, w, sw, bias, out_dtype=torch.float32)
    assert torch.equal(y, bias.expand(M, 6))


def check_linear(M, K, N, x_type, y_type, bias=True, seed=0, f=1.0):
    spread = torch.exp(normal(M, 1, seed=seed))
    x = T.quantize_mx4((normal(M, K, seed=seed + 1) * spread * f).to(x_type))
    w = T.quantize_mx4(normal(N, K, seed=seed + 2) / math.sqrt(max(K, 1)))
    b = normal(N, seed=seed + 3) if bias else None
    y = T.linear_mx4(*x, *w, b, out_dtype=y_type)
    xv, wv = values(*x), values(*w)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if b is not None:
        ref, size = ref + b.double(), size + b.double().abs()
    assert y.shape == (M, N) and y.dtype == y_type
    sums = (K + 1) * 2.0 ** -24 * size
    tol = HALF[y_type] * (ref.abs() + sums) + sums + TINY[y_type]
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    return x, w, b, y


SHAPES = [(1, 1, 1), (1, 1152, 3456), (2, 33, 7), (16, 640, 100), (17, 1152, 64), (33, 257, 1283),
          (64, 2240, 130), (65, 128, 63), (70, 1152, 65), (237, 640, 1283), (300, 77, 640),
          (256, 256, 256), (511, 384, 1160), (1000, 1153, 1152), (2048, 1152, 1152),
          (1500, 700, 9001)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("y_type", list(HALF))
def test_linear(M, K, N, y_type):
    check_linear(M, K, N, torch.bfloat16, y_type, seed=M + N)


@pytest.mark.parametrize("M,K,N", [(1, 640, 96), (65, 640, 96), (300, 4608, 1152), (8192, 640, 1160)])
def test_linear_without_bias(M, K, N):
    check_linear(M, K, N, torch.float32, torch.float32, bias=False)


@pytest.mark.parametrize("f", [2.0 ** -60, 2.0 ** 60])
def test_linear_of_far_scales(f):
    check_linear(20, 300, 70, torch.float32, torch.float32, bias=False, f=f)
    check_linear(90, 300, 70, torch.float32, torch.float32, bias=False, f=f)


def test_one_value_at_every_place():
    """Ones at one place of K against weights that name their place."""
    K = 384
    w = torch.zeros(K, K, device=DEV)
    at = torch.arange(K, device=DEV)
    w[at, at] = torch.tensor(GRID[1:], device=DEV)[at % 7] * 2.0 ** (at % 5)
    W = T.quantize_mx4(w)
    for M in (16, 64, 384):
        x = torch.zeros(M, K, device=DEV)
        rows = torch.arange(M, device=DEV)
        x[rows, (rows * 7 + 3) % K] = 2.0
        y = T.linear_mx4(*T.quantize_mx4(x), *W, out_dtype=torch.float32)
        assert torch.equal(y, x @ w.t())


@pytest.mark.parametrize("M", [3, 40, 200, 1000])
@pytest.mark.parametrize("N", [1283, 1288])
def test_output_between_other_data(M, N):
    """The output at an address of its elements only, nothing around it written."""
    x, w, b, y = check_linear(M, 256, N, torch.bfloat16, torch.bfloat16)
    flat = torch.full((M * N + 11,), 7.0, dtype=torch.bfloat16, device=DEV)
    got = T.linear_mx4(*x, *w, b, y=flat[3:3 + M * N].view(M, N))
    assert torch.equal(got, y)
    assert bool((flat[:3] == 7).all()) and bool((flat[3 + M * N:] == 7).all())


def test_more_than_two_gib():
    """Inputs past 2^31 elements, codes past 2^30: the last rows as alone."""
    M, K, N = 140000, 16384, 8
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    x[-3:] = normal(3, K, dtype=torch.bfloat16)
    X, sx = T.quantize_mx4(x)
    one = T.quantize_mx4(x[-3:].contiguous())
    assert torch.equal(X[-3:], one[0]) and torch.equal(sx[-3:], one[1])
    W = T.quantize_mx4(normal(N, K))
    ref = values(*one) @ values(*W).t()
    y = T.linear_mx4(X, sx, *W, out_dtype=torch.float32)
    size = values(*one).abs() @ values(*W).abs().t()
    assert bool(((y[-3:].double() - ref).abs() <= (K + 1) * 2.0 ** -24 * size).all())
    assert not y[:-3].any()
    del x
    # the other way round: many channels, few tokens
    y = T.linear_mx4(*W, X, sx, out_dtype=torch.float32)
    assert bool(((y[:, -3:].t().double() - ref).abs() <= (K + 1) * 2.0 ** -24 * size).all())


def test_wide_output():
    """An output of more than 2^32 bytes."""
    M, N = 70, 40_000_000
    x, w = T.quantize_mx4(normal(M, 32)), T.quantize_mx4(normal(1000, 32))
    W, sw = (t.repeat(N // 1000, 1) for t in w)
    y = T.linear_mx4(*x, W, sw)
    few = T.linear_mx4(*x, *w)
    assert torch.equal(y[:, :1000], few) and torch.equal(y[:, -1000:], few)


def test_captured_and_replayed():
    x = normal(200, 1152, dtype=torch.bfloat16)
    w = T.quantize_mx4(normal(640, 1152))

    def f():
        return T.linear_mx4(*T.quantize_mx4(x), *w)
    f()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = f()
    for seed in range(3):
        x.copy_(normal(200, 1152, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, f())
