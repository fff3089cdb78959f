"""Gradient of the token-scaled linear where the rows of codes are shorter than a
dword: the 8 bytes that a lane loads then reach over several rows, and past the
operand's end from rows of the last two steps of the sum.

Codes are one in the last few rows and zero before them, factors and gradients one, so
that every sum is a small whole number and exact in either type, in any order.
"""
import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"
LAST = 5


def check(M, N, K, dtype, offset=0):
    def codes(rows):
        flat = torch.zeros(rows * K + offset, dtype=torch.int8, device=DEV)
        q = flat[offset:].view(rows, K)
        q[-LAST:] = 1
        return q
    dy = torch.ones(M, N, dtype=dtype, device=DEV)
    one = [torch.ones(n, device=DEV) for n in (M, N)]
    dx, dw, dbias = T.masked_linear_tokens_backward(dy, codes(M), codes(N), *one, 8)
    for name, got, rows, terms in (("dx", dx, M, N), ("dw", dw, N, M)):
        assert torch.equal(got.float(), torch.full((rows, K), float(min(LAST, terms)), device=DEV)), \
            (name, got.float().unique())
    assert torch.equal(dbias, torch.full((N,), float(M), device=DEV))


@pytest.mark.parametrize("M", [1, 63, 64, 65, 66, 67, 128, 129, 130, 193])
@pytest.mark.parametrize("N", [1, 65, 66, 129])
@pytest.mark.parametrize("K", [1, 2, 3, 5])
def test_rows_of_few_codes(M, N, K):
    for dtype in (torch.bfloat16, torch.float16):
        check(M, N, K, dtype)
        check(N, M, K, dtype)


@pytest.mark.parametrize("K", [1, 2, 3])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_codes_at_any_address(K, offset):
    check(130, 65, K, torch.bfloat16, offset)


@pytest.mark.parametrize("M,N", [(64 * 130 + 1, 66), (64 * 130 + 2, 1281),  # ranges of the tokens
                                 (66, 64 * 130 + 1),                        # ranges of the channels
                                 (64 * 312 + 1, 64 * 40 + 1)])              # tiles of 128
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_sums_of_one_code(M, N, dtype):
    check(M, N, 1, dtype)


def test_one_gradient_of_one_by_row():
    """A gradient of one at each of the last rows of a sum picks that row's code."""
    M = N = 66
    X = torch.arange(1, M + 1, device=DEV).to(torch.int8).view(M, 1)
    W = (-X).contiguous()
    one = torch.ones(M, device=DEV)
    for at in (0, 61, 62, 63, 64, 65):
        dy = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV)
        dy[at, at] = 1.0
        dx, dw, _ = T.masked_linear_tokens_backward(dy, X, W, one, one, 8)
        assert dx[at] == -(at + 1) and dw[at] == at + 1
        assert dx.abs().sum() == at + 1 and dw.abs().sum() == at + 1
