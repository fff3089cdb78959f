"""Token-scaled linears with many tiles of 256x256 on the GPU: the persistent walk
and the launch of one tile to a workgroup that stands in where its 32-bit
offsets or 16-byte rows do not hold.  Bounds as for the small ones: at most
four fp32 roundings, 2^-22 (|acc sx sw| + |bias|), and half a unit in the last
place of a 16-bit output.  The products are taken in 64 bits, where they are
exact."""
import pytest
import torch

import paper_2608_03057_amd as T
from test_gpu_tokens import ROUND, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def problem(M, N, K, bias, seed=0, offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * M + 7 * N + K)
    X, W = (torch.empty(r * K + offset, dtype=torch.int8, device=DEV)[offset:].view(r, K)
            for r in (M, N))
    for t in (X, W):
        t.copy_(torch.randint(-128, 128, t.shape, generator=g, device=DEV, dtype=torch.int16))
    sx = torch.rand(M, generator=g, device=DEV) * 0.05
    sx[M // 3] = 0.0
    sw = torch.rand(N, generator=g, device=DEV) * 0.01
    return X, W, sx, sw, torch.randn(N, generator=g, device=DEV) if bias else None


def compare(y, X, W, sx, sw, b, bias, columns=1 << 16):
    """y against the definition, some columns at a time."""
    step = 2 ** (8 - b)
    X = X.double()
    for n in range(0, W.shape[0], columns):
        c = slice(n, n + columns)
        Wb = torch.floor(W[c].double() / step) * step
        prod = torch.matmul(X, Wb.t().contiguous()) * sx.double()[:, None] * sw[c].double()[None]
        bb = 0.0 if bias is None else bias[c].double()
        ref = prod + bb
        mag = prod.abs() + (0.0 if bias is None else bb.abs())
        tol = 2.0 ** -22 * mag + ROUND[y.dtype] * ref.abs() * (1 + 2.0 ** -10) + TINY[y.dtype]
        err = (y[:, c].double() - ref).abs()
        assert bool((err <= tol).all()), (n, float((err - tol).max()))


# 170 to 340 tiles: one, two and three or more K tiles of 128, whole and with a
# remainder; rows and columns off 256; more tiles than compute units, so that
# a workgroup goes from one to the next.
WALKS = [(4100, 4104, 16), (4100, 4104, 128), (2305, 4616, 144), (4100, 4104, 256),
         (4353, 4104, 272), (2305, 4616, 400), (4100, 4104, 1152), (8192, 2568, 640)]


@pytest.mark.parametrize("M,N,K", WALKS)
@pytest.mark.parametrize("dtype", TYPES)
def test_walk(M, N, K, dtype):
    b = 1 + (M + N + K // 16) % 8
    X, W, sx, sw, bias = problem(M, N, K, K % 256 != 0)
    y = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    T.masked_linear_tokens(X, W, sx, sw, b, bias, y=y)
    compare(y, X, W, sx, sw, b, bias)


@pytest.mark.parametrize("M,N,K,offset", [
    (2305, 4617, 400, 0),       # (fp32: the walk with rows at any 4 bytes)
    (2305, 4612, 384, 0), (2305, 4616, 151, 0), (2305, 4616, 1151, 0), (2305, 4616, 384, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_and_operands_off_the_alignment(M, N, K, offset, dtype):
    X, W, sx, sw, bias = problem(M, N, K, N % 8 != 0, offset=offset)
    y = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    T.masked_linear_tokens(X, W, sx, sw, 6, bias, y=y)
    compare(y, X, W, sx, sw, 6, bias)


@pytest.mark.parametrize("dtype", TYPES)
def test_output_off_sixteen_bytes(dtype):
    M, N, K = 2305, 4616, 272
    X, W, sx, sw, bias = problem(M, N, K, True)
    buf = torch.full((M * N + 9,), 99.0, dtype=dtype, device=DEV)
    y = buf[1:1 + M * N].view(M, N)
    T.masked_linear_tokens(X, W, sx, sw, 7, bias, y=y)
    compare(y, X, W, sx, sw, 7, bias)
    assert float(buf[0]) == 99.0 and bool((buf[1 + M * N:] == 99.0).all())


def test_walk_repeats_its_bits():
    X, W, sx, sw, bias = problem(4100, 4104, 640, True)
    y = [T.masked_linear_tokens(X, W, sx, sw, 5, bias) for _ in range(4)]
    assert all(torch.equal(y[0], t) for t in y[1:])


@pytest.mark.parametrize("N,dtype", [(4_300_000, torch.float32), (8_600_000, torch.bfloat16),
                                     (8_600_000, torch.float16)])
def test_rows_past_the_end_of_a_very_wide_output(N, dtype):
    """66 rows of a 256-row tile: 250 rows on, an offset of 32 bits in bytes would be
    back inside the output."""
    M, K = 66, 16
    assert M * N * dtype.itemsize < 2 ** 31 and 255 * N * dtype.itemsize > 2 ** 32
    X, W, sx, sw, bias = problem(M, N, K, True)
    y = T.masked_linear_tokens(X, W, sx, sw, 8, bias, out_dtype=dtype)
    compare(y, X, W, sx, sw, 8, bias)


@pytest.mark.parametrize("K", [0, 17])
def test_one_token_and_more_channels_than_a_launch_of_few_takes(K):
    """2^28 channels and some: 16 to a workgroup would be 2^32 threads."""
    N = (1 << 28) + 40
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    X, W, sx, sw, bias = problem(1, 64, K, True)
    sx += 0.01
    W, sw, bias = (t.repeat((N + 63) // 64, *[1] * (t.dim() - 1))[:N] for t in (W, sw, bias))
    y = T.masked_linear_tokens(X, W, sx, sw, 8, bias)
    compare(y[:, :4096], X, W[:4096], sx, sw[:4096], 8, bias[:4096])
    assert torch.equal(y[0, :N // 64 * 64].view(-1, 64), y[0, :64].expand(N // 64, 64))
    assert torch.equal(y[0, N // 64 * 64:], y[0, :N % 64])


@pytest.mark.parametrize("M,N,K", [(66000, 300, 32768), (300, 66000, 32768), (9, 66000, 32768)])
def test_operands_past_two_gigabytes(M, N, K):
    """More codes than a 32-bit byte offset reaches: the first, last and some rows."""
    X, W, sx, sw, bias = problem(M, N, K, True)
    y = T.masked_linear_tokens(X, W, sx, sw, 6, bias)
    m, n = (torch.cat([torch.arange(s - 200 if s > 400 else 0, s),
                       torch.arange(0, s, max(1, s // 150))]).to(DEV) for s in (M, N))
    compare(y[m][:, n], X[m].contiguous(), W[n].contiguous(), sx[m], sw[n], 6, bias[n])
