"""Sizes that the wrappers refuse before a call: an int of the C ABI would not hold
them, and the call would have another's.  (Expanded tensors: no memory.)"""
import pytest
import torch

import paper_2608_03057_amd as T

BIG = (1 << 32) + 3


def expanded(dtype, *shape):
    return torch.empty(1, dtype=dtype).expand(*shape)


@pytest.mark.parametrize("shape", [(BIG, 1), (1, BIG), (1 << 31, 1)])
def test_quantize_tokens(shape):
    with pytest.raises(ValueError, match="below 2\\^31"):
        T.quantize_tokens(expanded(torch.bfloat16, *shape))


@pytest.mark.parametrize("M,N,K", [(BIG, 1, 1), (1, BIG, 1), (1, 1, BIG)])
def test_masked_linear_tokens(M, N, K):
    with pytest.raises(ValueError, match="below 2\\^31"):
        T.masked_linear_tokens(expanded(torch.int8, M, K), expanded(torch.int8, N, K),
                               expanded(torch.float32, M), expanded(torch.float32, N), 8)
