"""Gradient of the token-scaled linear over much work, whatever the layout of dy: with
the workspace that the query asks for, the products are the same ones, so that the
results have the same bits as those of a contiguous dy."""
import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"


def make(M, N, K, dtype):
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    return [(0.3 * torch.randn(M, N, generator=g, device=DEV)).to(dtype),
            torch.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=torch.int8),
            torch.randint(-128, 128, (N, K), generator=g, device=DEV, dtype=torch.int8),
            0.01 * torch.exp(torch.randn(M, generator=g, device=DEV)),
            1e-3 + 4e-3 * torch.rand(N, generator=g, device=DEV)]


def layouts(dy):
    """dy at an odd address, at an odd distance of rows, and both; NaN around it."""
    M, N = dy.shape
    for first, width in ((5, N + 8), (0, N + 9), (3, N + 13)):
        wide = torch.full((M, width), float("nan"), dtype=dy.dtype, device=DEV)
        wide[:, first:first + N] = dy
        yield wide[:, first:first + N]


@pytest.mark.parametrize("M,N,K", [(520, 4456, 4408), (2048, 2240, 2400), (8195, 1152, 1160),
                                   (520, 4451, 4408)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_same_results_for_any_layout(M, N, K, dtype):
    dy, *rest = make(M, N, K, dtype)
    plain = T.masked_linear_tokens_backward(dy, *rest, 6)
    for other in layouts(dy):
        got = T.masked_linear_tokens_backward(other, *rest, 6)
        assert all(torch.equal(p, q) for p, q in zip(got, plain))
        only = T.masked_linear_tokens_backward(other, *rest, 6, need_input=False)
        assert torch.equal(only[1], plain[1]) and torch.equal(only[2], plain[2])
        only = T.masked_linear_tokens_backward(other, *rest, 6, need_weight=False)
        assert torch.equal(only[0], plain[0])


def test_workspace_of_the_query_is_all_that_is_written():
    M, N, K = 520, 4456, 4408
    dy, *rest = make(M, N, K, torch.bfloat16)
    n = T.masked_linear_tokens_backward_workspace_bytes(M, N, K)
    plain = T.masked_linear_tokens_backward(dy, *rest, 6)
    for other in layouts(dy):
        room = torch.full((n + 512,), 9, dtype=torch.uint8, device=DEV)
        got = T.masked_linear_tokens_backward(other, *rest, 6, workspace=room[:n])
        assert all(torch.equal(p, q) for p, q in zip(got, plain)) and bool((room[n:] == 9).all())
