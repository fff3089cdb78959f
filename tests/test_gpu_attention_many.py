"""Attention and its gradient with more workgroups than one launch takes (2^24 of 256
threads): 2^31 queries over two keys.  All of a batch entry's queries are the same
one, so that each row is known, and checked."""
import math

import pytest
import torch

import paper_2608_03057_amd as T
from test_gpu_attention import Exact, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def same_rows(t, want):
    """Whether all rows of t [1, S, 1, D] have the bits of want [D]."""
    step = 1 << 26
    return all(bool((t[:, i:i + step] == want).all()) for i in range(0, t.shape[1], step))


def test_more_workgroups_than_a_launch_takes():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB of device memory")
    B, SQ, SK, D, dtype = 2, 1 << 30, 2, 8, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(4)
    draw = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
    one, done, k, v = draw(B, 1, 1, D), draw(B, 1, 1, D), draw(B, SK, 1, D), draw(B, SK, 1, D)
    q, do = one.expand(B, SQ, 1, D), done.expand(B, SQ, 1, D)
    out = torch.full((B, SQ, 1, D), math.nan, dtype=dtype, device=DEV)
    lse = torch.full((B, 1, SQ), math.nan, device=DEV)
    T.attention(q, k, v, out=out, lse=lse)
    few, few_lse = T.attention(one, k, v, want_lse=True)
    near(few, *Exact(one, k, v).forward()[:2], "out")
    for b in range(B):
        assert same_rows(out[b:b + 1], few[b, 0, 0])
        assert bool((lse[b] == few_lse[b]).all())
    dq = torch.full((B, SQ, 1, D), math.nan, dtype=dtype, device=DEV)
    T.attention_backward(do, q, k, v, out, lse, dq=dq)
    few_dq = T.attention_backward(done, one, k, v, few, few_lse)[0]
    refs, tols = Exact(one, k, v).backward(done, few, few_lse)
    near(few_dq, refs[0], tols[0], "dq")
    for b in range(B):
        assert same_rows(dq[b:b + 1], few_dq[b, 0, 0])
    del out, lse, dq
    torch.cuda.empty_cache()
