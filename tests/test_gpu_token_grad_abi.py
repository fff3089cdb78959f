"""Calls of the token-scaled linear's gradient that only the C ABI allows: operands that
are not read may be NULL, the bias' gradient of a linear without input channels among
them."""
import pytest
import torch

from paper_2608_03057_amd import _lib

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {torch.bfloat16: _lib.TYPE_BF16, torch.float16: _lib.TYPE_F16}


def at(t):
    return None if t is None else t.data_ptr()


def call(dy, X, sx, W, sw, N, K, dx=None, dw=None, dbias=None, workspace=None):
    M = dy.shape[0]
    rc = _lib.lib().tasq_masked_linear_tokens_backward(
        at(dy), TYPES[dy.dtype], N, at(X), at(sx), at(W), at(sw), M, N, K, 8, at(dx), at(dw),
        at(dbias), at(workspace), 0 if workspace is None else workspace.numel(),
        torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("M,N", [(1, 1), (5, 64), (24, 16), (70, 129), (300, 1283), (5000, 40)])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cut", [False, True])
def test_bias_gradient_without_input_channels(M, N, dtype, cut):
    """Whole numbers, whose sums are exact in any order."""
    dy = (torch.arange(M * N, device=DEV) % 15 - 7).view(M, N).to(dtype)
    dbias = torch.full((N,), 9.0, device=DEV)
    n = _lib.lib().tasq_masked_linear_tokens_backward_workspace_bytes(M, N, 0) if cut else 0
    ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    call(dy, None, None, None, None, N, 0, dbias=dbias, workspace=ws)
    assert torch.equal(dbias, dy.float().sum(0))


@pytest.mark.parametrize("M,N,K", [(70, 136, 96), (65, 71, 33), (520, 4456, 4408)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_operands_that_are_not_read(M, N, K, dtype):
    g = torch.Generator(device=DEV).manual_seed(M)
    dy = torch.randn(M, N, generator=g, device=DEV).to(dtype)
    X = torch.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=torch.int8)
    W = torch.randint(-128, 128, (N, K), generator=g, device=DEV, dtype=torch.int8)
    sx, sw = (torch.rand(n, generator=g, device=DEV) for n in (M, N))
    n = _lib.lib().tasq_masked_linear_tokens_backward_workspace_bytes(M, N, K)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)

    def outputs():
        return (torch.empty(M, K, dtype=dtype, device=DEV),
                torch.empty(N, K, dtype=dtype, device=DEV), torch.empty(N, device=DEV))
    both, one = outputs(), outputs()
    call(dy, X, sx, W, sw, N, K, *both, workspace=ws)
    call(dy, None, None, W, sw, N, K, dx=one[0], workspace=ws)
    call(dy, X, sx, None, None, N, K, dw=one[1], dbias=one[2], workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(both, one))
