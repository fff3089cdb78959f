"""Gradient of the token-scaled linear against its formula in 64 bits.

Tolerances: the 8-bit operand times its factor is rounded once to dy's type (half a
step of each product's magnitude), the sums over Z round to fp32 (at most Z half
steps of 2^-24 of the products' magnitudes, over ranges as well), the result is
rounded once.  In half a product next to the least numbers is off by half of 2^-24 of
a unit that is at most 2^-7 of the largest factor: 2^-32 of it.
"""
import math

import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
BOTH = list(HALF)


def make(M, N, K, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return dict(
        dy=(0.3 * torch.randn(M, N, generator=g, device=DEV)).to(dtype),
        X=torch.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=torch.int8),
        W=torch.randint(-128, 128, (N, K), generator=g, device=DEV, dtype=torch.int8),
        sx=0.01 * torch.exp(torch.randn(M, generator=g, device=DEV)),
        sw=1e-3 + 4e-3 * torch.rand(N, generator=g, device=DEV))


def masked(W, b):
    return torch.bitwise_and(W.to(torch.int32), -(1 << (8 - b))).double()


def product(A, s, Q, dtype):
    """(A diag(s) Q in 64 bits, its error before the last rounding)"""
    A, v = A.double(), s.double()[:, None] * Q
    size = A.abs() @ v.abs()
    err = (HALF[dtype] + (Q.shape[0] + 2) * 2.0 ** -24) * size
    if dtype == torch.float16 and len(s):
        err += 2.0 ** -32 * float(s.abs().max()) * A.abs().sum(1, keepdim=True)
    return A @ v, err


def close(got, ref, err, dtype, name):
    assert got.dtype == dtype and got.shape == ref.shape, name
    half = HALF.get(dtype, 2.0 ** -24)
    tol = half * (ref.abs() + err) + err + TINY.get(dtype, 0.0)
    off = (got.double() - ref).abs()
    assert bool((off <= tol).all()), (name, float((off / tol.clamp(min=1e-300)).max()))


def check(a, b, **kw):
    dtype = a["dy"].dtype
    dx, dw, dbias = T.masked_linear_tokens_backward(a["dy"], a["X"], a["W"], a["sx"], a["sw"], b,
                                                    **kw)
    if dx is not None:
        close(dx, *product(a["dy"], a["sw"], masked(a["W"], b), dtype), dtype, "dx")
    if dw is not None:
        close(dw, *product(a["dy"].t(), a["sx"], a["X"].double(), dtype), dtype, "dw")
        dy = a["dy"].double()
        close(dbias, dy.sum(0), (len(dy) + 2) * 2.0 ** -24 * dy.abs().sum(0), torch.float32, "dbias")
    return dx, dw, dbias


SHAPES = [(1, 1, 1), (1, 8, 16), (1, 1152, 640), (2, 7, 33), (7, 64, 64), (16, 1152, 1152),
          (63, 65, 17), (64, 64, 64), (65, 128, 80), (100, 1283, 640), (130, 200, 129),
          (300, 1283, 641), (256, 256, 256), (257, 264, 272), (520, 1000, 1153), (2048, 640, 1152),
          (1100, 2056, 1160), (5000, 48, 32), (48, 5000, 32), (4097, 130, 48)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", BOTH)
def test_sizes(M, N, K, dtype):
    check(make(M, N, K, dtype, M + N), 8)


@pytest.mark.parametrize("N", range(257, 264))
@pytest.mark.parametrize("dtype", BOTH)
def test_rows_that_end_inside_a_chunk_over_many_tokens(N, dtype):
    check(make(513, N, 130, dtype, N), 8)


@pytest.mark.parametrize("M,N,K", [(700, 1283, 640), (1001, 1000, 129), (2049, 513, 1001),
                                   (1283, 2051, 641)])
@pytest.mark.parametrize("dtype", BOTH)
def test_odd_sizes_over_many_tokens(M, N, K, dtype):
    check(make(M, N, K, dtype, M + N), 8)


@pytest.mark.parametrize("M,N,K", [(512, 4449, 4400), (513, 4450, 4401), (515, 4451, 4402),
                                   (519, 4453, 4403), (520, 4455, 4407), (2049, 2563, 2001),
                                   (8195, 1153, 1100)])
@pytest.mark.parametrize("dtype", BOTH)
def test_odd_sizes_of_much_work(M, N, K, dtype):
    check(make(M, N, K, dtype, M + N), 8)


@pytest.mark.parametrize("N,K", [(1, 1), (1, 2), (2, 1), (3, 1), (1, 5), (5, 3), (6, 7), (9, 9)])
@pytest.mark.parametrize("M", [1, 2, 3, 66])
def test_rows_of_less_than_a_chunk(M, N, K):
    """Chunks of these reach over many rows, and past the last one."""
    check(make(M, N, K, torch.bfloat16, M), 8)


@pytest.mark.parametrize("b", range(1, 9))
def test_bits(b):
    check(make(70, 136, 96, torch.bfloat16), b)


@pytest.mark.parametrize("M,N,K", [(8192, 1152, 1152), (4096, 2240, 2240), (3000, 3456, 1152)])
def test_large(M, N, K):
    check(make(M, N, K, torch.bfloat16), 6)


@pytest.mark.parametrize("dtype", BOTH)
def test_one_at_every_place(dtype):
    """A single gradient of one picks a row of the weight and of the codes."""
    for M, N, K in ((300, 264, 272), (65, 72, 80)):
        a = make(M, N, K, dtype)
        a["sx"].fill_(0.5)
        a["sw"].fill_(0.25)
        for m, n in ((0, 0), (M - 1, N - 1), (M // 2, 17), (33, N // 2)):
            a["dy"].zero_()
            a["dy"][m, n] = 1.0
            dx, dw, dbias = T.masked_linear_tokens_backward(a["dy"], a["X"], a["W"], a["sx"],
                                                            a["sw"], 8)
            assert torch.equal(dx[m].float(), 0.25 * a["W"][n].float())
            assert torch.equal(dw[n].float(), 0.5 * a["X"][m].float())
            dx[m], dw[n] = 0, 0
            assert not dx.any() and not dw.any()
            assert dbias[n] == 1 and dbias.abs().sum() == 1


def test_parts_of_the_result():
    a = make(90, 72, 48, torch.bfloat16)
    args = [a[n] for n in ("dy", "X", "W", "sx", "sw")]
    both = check(a, 5)
    dx, dw, dbias = check(a, 5, need_weight=False)
    assert dw is None and dbias is None and torch.equal(dx, both[0])
    dx, dw, dbias = check(a, 5, need_input=False)
    assert dx is None and torch.equal(dw, both[1]) and torch.equal(dbias, both[2])
    assert T.masked_linear_tokens_backward(*args, 5, need_input=False,
                                           need_weight=False) == (None,) * 3
    outs = [torch.full_like(t, 9) for t in both]
    got = T.masked_linear_tokens_backward(*args, 5, dx=outs[0], dw=outs[1], dbias=outs[2])
    assert all(p is q and torch.equal(p, r) for p, q, r in zip(got, outs, both))


@pytest.mark.parametrize("M,N,K", [(0, 24, 16), (24, 0, 16), (24, 16, 0), (0, 0, 0)])
def test_nothing(M, N, K):
    a = make(M, N, K, torch.bfloat16)
    dx, dw, dbias = check(a, 8)
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("M,N,K", [(300, 136, 144), (2500, 72, 80), (131, 63, 49)])
def test_strided_rows_and_offset_outputs(M, N, K):
    a = make(M, N, K, torch.float16)
    plain = check(a, 7)
    wide = torch.full((M, N + 9), math.nan, dtype=torch.float16, device=DEV)
    wide[:, 5:5 + N] = a["dy"]
    even = torch.full((M, N + 8), math.nan, dtype=torch.float16, device=DEV)
    even[:, :N] = a["dy"]
    for dy in (wide[:, 5:5 + N], even[:, :N]):
        check({**a, "dy": dy}, 7)
    # codes and outputs at addresses of their elements only, nothing written around
    flat = torch.zeros(M * K + 3, dtype=torch.int8, device=DEV)
    X = flat[3:].view(M, K)
    X.copy_(a["X"])
    room = torch.full((M * K + 11,), 7.0, dtype=torch.float16, device=DEV)
    got = check({**a, "X": X}, 7, dx=room[3:3 + M * K].view(M, K))
    assert torch.equal(got[0], plain[0])
    assert bool((room[:3] == 7).all()) and bool((room[3 + M * K:] == 7).all())


def test_without_workspace():
    """Ranges uncut: a workspace too small for them, and the parts' sums agree."""
    a = make(4096, 128, 256, torch.bfloat16)
    assert T.masked_linear_tokens_backward_workspace_bytes(4096, 128, 256) > 256
    check(a, 8)
    check(a, 8, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("small", [1e-3, 1e-6, 2.0 ** -40])
def test_half_of_small_factors(small):
    """Scales far below half's range, and tokens of very different sizes."""
    a = make(200, 72, 80, torch.float16)
    a["sx"] *= small
    a["sw"] *= small
    check(a, 8)
    a["sx"][::3] *= 2.0 ** -12
    check(a, 8)


def test_half_of_large_factors():
    a = make(200, 72, 80, torch.float16)
    a["sx"] *= 1e5
    a["dy"] *= 1e-3
    check(a, 8)


@pytest.mark.parametrize("dtype", BOTH)
def test_zero_scales(dtype):
    a = make(200, 72, 80, dtype)
    a["sx"][5] = 0.0
    check(a, 8)
    a["sx"].zero_()
    a["sw"].zero_()
    dx, dw, _ = check(a, 8)
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", BOTH)
def test_values_that_are_not_finite(bad, dtype):
    """A gradient that is not finite stays in its token's dx and its channel's dw; a
    token of such a scale reaches all of dw and nothing of dx."""
    a = make(300, 136, 144, dtype)
    dx, dw, dbias = check(a, 8)
    args = [a[n] for n in ("dy", "X", "W", "sx", "sw")]
    args[0] = a["dy"].clone()
    args[0][70, 9] = bad
    gx, gw, gb = T.masked_linear_tokens_backward(*args, 8)
    rows, channels = torch.arange(300, device=DEV) != 70, torch.arange(136, device=DEV) != 9
    assert torch.equal(gx[rows], dx[rows]) and torch.equal(gw[channels], dw[channels])
    assert torch.equal(gb[channels], dbias[channels]) and not torch.isfinite(gb[9])
    assert not torch.isfinite(gx[70]).any() and not torch.isfinite(gw[9]).any()
    args[0] = a["dy"]
    args[3] = a["sx"].clone()
    args[3][70] = bad
    args[1] = a["X"].clone()
    args[1][70] = 5
    gx, gw, gb = T.masked_linear_tokens_backward(*args, 8)
    assert torch.equal(gx, dx) and torch.equal(gb, dbias) and not torch.isfinite(gw).any()


def test_differences_of_the_forward_pass():
    """One code more is sx[m] more of an activation: the linear's outputs at both
    (exact sums, fp32 out) give that element of dx.  fp32: two products and a sum each,
    of outputs that the difference is small against."""
    a = make(40, 72, 96, torch.bfloat16)
    b, dy = 6, a["dy"].double()
    dx, _, _ = check(a, b)

    def outputs(X):
        return T.masked_linear_tokens(X, a["W"], a["sx"], a["sw"], b,
                                      out_dtype=torch.float32).double()
    base = outputs(a["X"])
    for m, k in ((0, 0), (39, 95), (17, 40)):
        X = a["X"].clone()
        step = 1 if X[m, k] < 100 else -1
        X[m, k] += step
        moved = outputs(X)
        got = float((dy * (moved - base)).sum()) * step / float(a["sx"][m])
        slack = float((dy.abs() * (moved.abs() + base.abs())).sum()) * 3 * 2.0 ** -24
        _, err = product(a["dy"][m:m + 1], a["sw"], masked(a["W"], b), torch.bfloat16)
        want = float(dx[m, k])
        assert abs(got - want) <= slack / float(a["sx"][m]) + float(err[0, k]) + \
            2.0 ** -8 * abs(want) * 1.01


def test_same_bits_each_time():
    a = make(4096, 264, 272, torch.bfloat16)
    args = [a[n] for n in ("dy", "X", "W", "sx", "sw")]
    first = T.masked_linear_tokens_backward(*args, 8)
    for _ in range(3):
        again = T.masked_linear_tokens_backward(*args, 8)
        assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_captured_and_replayed():
    a = make(700, 264, 272, torch.bfloat16)
    args = [a[n] for n in ("dy", "X", "W", "sx", "sw")]

    def f():
        return T.masked_linear_tokens_backward(*args, 7)
    f()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    for seed in range(3):
        new = make(700, 264, 272, torch.bfloat16, seed + 3)
        a["dy"].copy_(new["dy"])
        a["X"].copy_(new["X"])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, f()))


def test_more_than_two_gib():
    """A gradient of more than 2^31 elements: the last tokens' results as alone."""
    M, N, K = 1_050_000, 2056, 16
    a = make(64, N, K, torch.bfloat16)
    dy = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV)
    X = torch.zeros(M, K, dtype=torch.int8, device=DEV)
    sx = torch.ones(M, device=DEV)
    dy[-64:], X[-64:], sx[-64:] = a["dy"], a["X"], a["sx"]
    dx, dw, dbias = T.masked_linear_tokens_backward(dy, X, a["W"], sx, a["sw"], 8)
    assert not dx[:-64].any()
    close(dx[-64:].clone(), *product(a["dy"], a["sw"], masked(a["W"], 8), torch.bfloat16),
          torch.bfloat16, "dx")
    close(dw, *product(a["dy"].t(), a["sx"], a["X"].double(), torch.bfloat16), torch.bfloat16, "dw")
    d = a["dy"].double()
    close(dbias, d.sum(0), 70 * 2.0 ** -24 * d.abs().sum(0), torch.float32, "dbias")


# Much work: the codes become values first, in rows of whole cache lines.
MUCH = (520, 4456, 4408)


def arguments(a):
    return [a[n] for n in ("dy", "X", "W", "sx", "sw")]


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("N", [4456, 4451])
def test_much_work_with_values_that_are_not_finite(bad, N):
    M, _, K = MUCH
    a = make(M, N, K, torch.bfloat16)
    dx, dw, dbias = check(a, 8)
    args = arguments(a)
    args[0] = a["dy"].clone()
    args[0][300, N - 1] = bad
    gx, gw, gb = T.masked_linear_tokens_backward(*args, 8)
    rows = torch.arange(M, device=DEV) != 300
    assert torch.equal(gx[rows], dx[rows]) and torch.equal(gw[:-1], dw[:-1])
    assert torch.equal(gb[:-1], dbias[:-1]) and not torch.isfinite(gb[-1])
    assert not torch.isfinite(gx[300]).any() and not torch.isfinite(gw[-1]).any()
    args = arguments(a)
    args[3] = a["sx"].clone()
    args[3][M - 1] = bad
    args[1] = a["X"].clone()
    args[1][M - 1] = 5
    gx, gw, gb = T.masked_linear_tokens_backward(*args, 8)
    assert torch.equal(gx, dx) and torch.equal(gb, dbias) and not torch.isfinite(gw).any()


def test_much_work_in_half_of_far_factors():
    a = make(*MUCH, torch.float16)
    for small in (1e-6, 2.0 ** -40):
        check({**a, "sx": a["sx"] * small, "sw": a["sw"] * small}, 8)
    a["sx"][::3] *= 2.0 ** -12
    check(a, 8)
    a["sx"] *= 1e5
    check({**a, "dy": a["dy"] * 1e-3}, 8)
    a["sx"].zero_()
    dx, dw, _ = check(a, 8)
    assert dx.any() and not dw.any()


@pytest.mark.parametrize("N", [4456, 4455])
def test_much_work_of_strided_rows_and_offset_outputs(N):
    M, _, K = MUCH
    a = make(M, N, K, torch.bfloat16)
    plain = check(a, 7)
    wide = torch.full((M, N + 9), math.nan, dtype=torch.bfloat16, device=DEV)
    wide[:, 5:5 + N] = a["dy"]
    even = torch.full((M, N + 16 - N % 8), math.nan, dtype=torch.bfloat16, device=DEV)
    even[:, :N] = a["dy"]
    for dy in (wide[:, 5:5 + N], even[:, :N]):
        check({**a, "dy": dy}, 7)
    flat = torch.zeros(M * K + 3, dtype=torch.int8, device=DEV)
    X = flat[3:].view(M, K)
    X.copy_(a["X"])
    rooms = [torch.full((r * K + 11,), 7.0, dtype=torch.bfloat16, device=DEV) for r in (M, N)]
    got = check({**a, "X": X}, 7, dx=rooms[0][3:3 + M * K].view(M, K),
                dw=rooms[1][5:5 + N * K].view(N, K))
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    for room, first, n in ((rooms[0], 3, M * K), (rooms[1], 5, N * K)):
        assert bool((room[:first] == 7).all()) and bool((room[first + n:] == 7).all())


@pytest.mark.parametrize("M,N,K", [MUCH, (2048, 4453, 1160), (9000, 1152, 1000)])
def test_much_work_in_parts(M, N, K):
    """One result alone, and workspaces without room for the values or for the ranges."""
    a = make(M, N, K, torch.bfloat16)
    both = check(a, 6)
    dx, _, _ = check(a, 6, need_weight=False)
    assert torch.equal(dx, both[0])
    _, dw, dbias = check(a, 6, need_input=False)
    assert torch.equal(dw, both[1]) and torch.equal(dbias, both[2])
    n = T.masked_linear_tokens_backward_workspace_bytes(M, N, K)
    for part in (n // 2, 256):
        check(a, 6, workspace=torch.empty(part, dtype=torch.uint8, device=DEV))
    # (Bytes behind the workspace asked for stay.)
    room = torch.full((n + 512,), 9, dtype=torch.uint8, device=DEV)
    again = check(a, 6, workspace=room[:n])
    assert all(torch.equal(p, q) for p, q in zip(again, both)) and bool((room[n:] == 9).all())


@pytest.mark.parametrize("dtype", BOTH)
def test_much_work_captured_and_replayed(dtype):
    a = make(*MUCH, dtype)
    args = arguments(a)

    def f():
        return T.masked_linear_tokens_backward(*args, 7)
    f()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    for seed in range(3):
        new = make(*MUCH, dtype, seed + 3)
        for n in ("dy", "X", "sx"):
            a[n].copy_(new[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, f()))


def test_much_work_of_more_than_two_gib():
    M, N, K = 1_050_000, 2056, 256
    a = make(64, N, K, torch.bfloat16)
    dy = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV)
    X = torch.zeros(M, K, dtype=torch.int8, device=DEV)
    sx = torch.ones(M, device=DEV)
    dy[-64:], X[-64:], sx[-64:] = a["dy"], a["X"], a["sx"]
    dx, dw, dbias = T.masked_linear_tokens_backward(dy, X, a["W"], sx, a["sw"], 8)
    assert not dx[:-64].any()
    close(dx[-64:].clone(), *product(a["dy"], a["sw"], masked(a["W"], 8), torch.bfloat16),
          torch.bfloat16, "dx")
    close(dw, *product(a["dy"].t(), a["sx"], a["X"].double(), torch.bfloat16), torch.bfloat16, "dw")
    d = a["dy"].double()
    close(dbias, d.sum(0), 70 * 2.0 ** -24 * d.abs().sum(0), torch.float32, "dbias")
