"""Activation codes and linears of tokens that hold NaN or infinity: such a token's
scale, and with it all its outputs, are not finite either, and the other tokens
keep theirs."""
import math

import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("K", [5, 320, 1152, 3000, 9001, 20001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_broken_tokens(K, dtype):
    g = torch.Generator().manual_seed(K)
    x = torch.randn(9, K, generator=g).to(dtype).to(DEV)
    clean_q, clean_s = T.quantize_tokens(x)
    x[1, K // 2] = math.nan
    x[3, 0] = math.inf
    x[4, K - 1] = -math.inf
    x[6, K - 1], x[6, 0] = math.nan, math.inf
    x[7] = -math.nan
    q, s = T.quantize_tokens(x)
    assert bool(s[[1, 6, 7]].isnan().all())
    assert torch.equal(s[[3, 4]], torch.full((2,), math.inf, device=DEV))
    keep = [0, 2, 5, 8]
    assert torch.equal(q[keep], clean_q[keep]) and torch.equal(s[keep], clean_s[keep])
    W = torch.randint(-128, 128, (33, K), generator=g, dtype=torch.int16).to(torch.int8).to(DEV)
    sw = torch.rand(33, generator=g).to(DEV) + 0.1
    y = T.masked_linear_tokens(q, W, s, sw, 8, out_dtype=torch.float32)
    want = T.masked_linear_tokens(clean_q, W, clean_s, sw, 8, out_dtype=torch.float32)
    assert bool(y[[1, 6, 7]].isnan().all()) and not bool(y[[3, 4]].isfinite().any())
    assert torch.equal(y[keep], want[keep])
