"""Token-scaled linears on the GPU against the definition in exact integers
and 64 bits.

Codes and scales are decided in single precision by definition, so they are
compared bit for bit.  Outputs: y = fl(acc) * fl(sx sw) + bias takes at most
four roundings of 2^-24 relative to the larger of the product and the bias
(the conversion of acc, two products and the sum), so 2^-22 (|acc sx sw| +
|bias|) bounds them, and a 16-bit output adds half a unit in its last place,
2^-8 (bfloat16) or 2^-11 (half) of |y|, or half of half's smallest step."""
import numpy as np
import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUND = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def codes_of(x):
    """Codes and scales of fp32 numpy rows, by the definition."""
    x = x.astype(np.float32)
    top = np.abs(x).max(axis=1, initial=0.0).astype(np.float32)
    s = (top * np.float32(1.0 / 127.0)).astype(np.float32)
    q = np.zeros(x.shape, np.float32)
    some = s > 0
    with np.errstate(over="ignore"):
        q[some] = np.clip(np.rint((x[some] / s[some, None]).astype(np.float32)), -127, 127)
    return q.astype(np.int8), s


@pytest.mark.parametrize("M,K", [(1, 1), (3, 8), (5, 72), (2, 511), (7, 1152), (130, 640),
                                 (4, 2240), (3, 4104), (2, 9000), (2, 20000), (1, 131071)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_codes(M, K, dtype):
    g = torch.Generator().manual_seed(M * 1000 + K)
    x = torch.randn(M, K, generator=g) * torch.exp(3 * torch.randn(M, 1, generator=g))
    x[M // 2] = 0.0                                 # a token of zeros
    x = x.to(dtype)
    q, s = T.quantize_tokens(x.to(DEV))
    rq, rs = codes_of(x.float().numpy())
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)


def test_codes_of_extreme_and_tied_values():
    rows = np.zeros((6, 128), np.float32)
    rows[0] = np.linspace(-127, 127, 128)           # scale 1: ties at the halves
    rows[0, 5:9] = (0.5, 1.5, -2.5, -0.5)
    rows[1] = 2.0 ** -149 * np.arange(128)          # denormals
    rows[2] = 2.0 ** -149                           # a scale that vanishes
    rows[3] = np.float32(3e38) * np.linspace(-1, 1, 128).astype(np.float32)
    rows[4] = np.float32(1e-30) * np.linspace(-1, 1, 128).astype(np.float32)
    rows[5, 7] = -5.0
    q, s = T.quantize_tokens(torch.from_numpy(rows).to(DEV))
    rq, rs = codes_of(rows)
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_strided_and_offset_rows(dtype):
    buf = torch.randn(9, 3 * 640 + 3, device=DEV).to(dtype)
    for lo, hi in ((0, 640), (640, 1280), (1, 641), (3, 700)):
        x = buf[::2, lo:hi]
        q, s = T.quantize_tokens(x)
        rq, rs = codes_of(x.float().cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)


def check_linear(M, N, K, b, dtype, bias=True, seed=0, offset=0):
    g = torch.Generator().manual_seed(seed + 31 * M + 7 * N + K)
    X = torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int64).to(torch.int8)
    W = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int64).to(torch.int8)
    sx = torch.rand(M, generator=g) * 0.05
    sx[M // 3] = 0.0
    sw = torch.rand(N, generator=g) * 0.01
    bb = torch.randn(N, generator=g) if bias else None
    dev = [torch.empty(t.numel() + offset, dtype=t.dtype, device=DEV)[offset:].view(t.shape)
           for t in (X, W)]
    for d, t in zip(dev, (X, W)):
        d.copy_(t)
    y = T.masked_linear_tokens(dev[0], dev[1], sx.to(DEV), sw.to(DEV), b,
                               None if bb is None else bb.to(DEV), out_dtype=dtype)
    step = 2 ** (8 - b)
    Wb = torch.div(W.to(torch.float64), step, rounding_mode="floor") * step
    acc = X.to(torch.float64) @ Wb.t()              # exact: below 2^53
    prod = acc * sx.double()[:, None] * sw.double()[None]
    ref = prod + (0.0 if bb is None else bb.double())
    mag = prod.abs() + (0.0 if bb is None else bb.double().abs())
    tol = 2.0 ** -22 * mag + ROUND[dtype] * ref.abs() * (1 + 2.0 ** -10) + TINY[dtype]
    err = (y.cpu().double() - ref).abs()
    assert y.dtype == dtype
    assert bool((err <= tol).all()), float((err - tol).max())


SHAPES = [(1, 1, 1), (1, 3456, 1152), (2, 33, 640), (5, 1283, 77), (16, 640, 2048),
          (33, 96, 4096), (64, 1152, 1152), (65, 130, 129), (237, 1283, 640), (300, 200, 304),
          (129, 1, 1152), (1024, 1152, 1152), (700, 2240, 2240), (2048, 2312, 320)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_linear(M, N, K, dtype):
    check_linear(M, N, K, 8 if M % 2 else 5, dtype, bias=N % 2 == 0)


@pytest.mark.parametrize("b", range(1, 9))
@pytest.mark.parametrize("M", [1, 200])
def test_linear_bits(M, b):
    check_linear(M, 160, 352, b, torch.float32)


@pytest.mark.parametrize("M,N,K", [(3, 65, 1152), (200, 300, 1151), (513, 1024, 1152)])
def test_linear_unaligned_operands(M, N, K):
    check_linear(M, N, K, 6, torch.bfloat16, offset=3)


def test_linear_without_a_sum():
    bias = torch.randn(40, device=DEV)
    y = T.masked_linear_tokens(torch.empty(3, 0, dtype=torch.int8, device=DEV),
                               torch.empty(40, 0, dtype=torch.int8, device=DEV),
                               torch.ones(3, device=DEV), torch.ones(40, device=DEV), 8, bias,
                               out_dtype=torch.float32)
    assert torch.equal(y, bias.expand(3, 40))


def test_linear_at_the_int32_limit():
    """K = 131071 codes of -128 on both sides: the largest sum of the ABI."""
    K = 131071
    X = torch.full((2, K), -128, dtype=torch.int8, device=DEV)
    y = T.masked_linear_tokens(X, X[:1].clone(), torch.ones(2, device=DEV),
                               torch.ones(1, device=DEV), 8, out_dtype=torch.float32)
    assert torch.equal(y.cpu().double(), torch.full((2, 1), float(np.float32(K * 16384.0)),
                                                    dtype=torch.float64))


def test_empty_calls_write_nothing():
    q, s = T.quantize_tokens(torch.empty(0, 64, device=DEV))
    assert q.shape == (0, 64) and s.shape == (0,)
    y = torch.full((2, 0), 7.0, device=DEV)
    T.masked_linear_tokens(torch.ones(2, 16, dtype=torch.int8, device=DEV),
                           torch.ones(0, 16, dtype=torch.int8, device=DEV),
                           torch.ones(2, device=DEV), torch.ones(0, device=DEV), 8, y=y)
    torch.cuda.synchronize()


def test_refusals_of_the_wrappers():
    x = torch.randn(4, 64, device=DEV)
    with pytest.raises(ValueError):
        T.quantize_tokens(x.double())
    with pytest.raises(ValueError):
        T.quantize_tokens(x.t())
    with pytest.raises(ValueError):
        T.quantize_tokens(x.cpu())
    q, s = T.quantize_tokens(x)
    W, sw = torch.zeros(8, 64, dtype=torch.int8, device=DEV), torch.ones(8, device=DEV)
    with pytest.raises(T.TasqError):
        T.masked_linear_tokens(q, W, s, sw, 9)
    with pytest.raises(ValueError):
        T.masked_linear_tokens(q, W[:, :32].contiguous(), s, sw, 8)
    with pytest.raises(ValueError):
        T.masked_linear_tokens(q, W, s[:3], sw, 8)
    with pytest.raises(ValueError):
        T.masked_linear_tokens(q, W, s, sw, 8, out_dtype=torch.float64)


def test_codes_of_more_rows_than_one_launch_takes():
    """2^22 rows go out together; the rows behind them have their own codes."""
    M, K = (1 << 22) + 5, 3
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(M, K, generator=g, device=DEV)
    q, s = T.quantize_tokens(x)
    for rows in (slice(0, 7), slice((1 << 22) - 3, M)):
        want_q, want_s = T.quantize_tokens(x[rows].contiguous())
        assert torch.equal(q[rows], want_q) and torch.equal(s[rows], want_s)
    top = x.abs().amax(1)
    assert torch.equal(s, top * torch.tensor(1 / 127, dtype=torch.float32, device=DEV))
    assert int(q.abs().amax(1).min()) == 127


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", [1, 7, 9, 515, 1025, 2049, 4097, 16383, 16391])
def test_codes_at_any_length_and_offset(dtype, K):
    """Every path of a row's length, rows and codes off the vector alignment."""
    g = torch.Generator().manual_seed(K)
    buf = torch.randn(3, K + 2, generator=g).to(dtype).to(DEV)
    x = buf[:, 1:K + 1]
    out = torch.full((3 * K + 2,), 99, dtype=torch.int8, device=DEV)
    q, s = T.quantize_tokens(x, out[1:-1].view(3, K))
    want_q, want_s = T.quantize_tokens(x.float().contiguous())
    assert torch.equal(q, want_q) and torch.equal(s, want_s)
    assert int(out[0]) == 99 and int(out[-1]) == 99
    x64 = x.double()
    sx = (x64.abs().amax(1).float() * torch.tensor(1 / 127, device=DEV)).double()
    r = x64 / sx[:, None]
    assert torch.equal(s.double(), sx)
    # round(x / s) decided in fp32: a code next to the quotient by 1/2 and 2^-16 at most
    assert float((q.double() - r).abs().max()) <= 0.5 + 2.0 ** -16


@pytest.mark.parametrize("M", [1, 3, 8])
@pytest.mark.parametrize("K", [16, 17, 31, 63, 64, 65, 127, 255, 257, 1151, 2063, 4607])
def test_linear_of_few_tokens_at_any_length(M, K):
    check_linear(M, 71, K, 7, torch.float32, offset=K % 4)


def test_linear_reads_no_byte_past_its_operands():
    """Rows end where the allocation does, codes behind them change nothing."""
    K, N, M = 1151, 33, 5
    g = torch.Generator().manual_seed(12)
    buf = torch.randint(-128, 128, (2, M * K + N * K + 64), generator=g,
                        dtype=torch.int64).to(torch.int8).to(DEV)
    buf[1] = buf[0]
    buf[1, M * K:M * K + 32] = 77               # behind X
    buf[1, M * K + 32 + N * K:] = -55           # behind W
    y = [T.masked_linear_tokens(r[:M * K].view(M, K), r[M * K + 32:M * K + 32 + N * K].view(N, K),
                                torch.ones(M, device=DEV), torch.ones(N, device=DEV), 8,
                                out_dtype=torch.float32) for r in buf]
    assert torch.equal(y[0], y[1])
