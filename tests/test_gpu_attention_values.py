"""Attention on values and gradients at the ends of bfloat16's range.  Bounds as in
test_gpu_attention."""
import math

import pytest
import torch

import paper_2608_03057_amd as T
from test_gpu_attention import Exact, draw, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def aligned_scores(shape, height, dtype=torch.bfloat16):
    """Queries and keys whose scores are all about `height`."""
    q, k, v, do, _ = draw(*shape, dtype, size=0.02)
    D = shape[-1]
    side = math.sqrt(abs(height)) * D ** -0.25
    q = q + side
    k = k + math.copysign(side, height)
    return q.to(dtype), k.to(dtype), v, do


@pytest.mark.parametrize("shape", [(1, 40, 90, 2, 2, 64), (1, 3, 700, 4, 1, 72),
                                   (8, 300, 130, 25, 25, 40)])
@pytest.mark.parametrize("height", [10.0, 30.0, -30.0])
def test_large_values(shape, height):
    """Values of 2^100 and scores of 30: outputs of 2^100, not infinity."""
    q, k, v, _ = aligned_scores(shape, height)
    v = (v.float() * 2.0 ** 100).to(torch.bfloat16)
    ex = Exact(q, k, v)
    out, lse = T.attention(q, k, v, want_lse=True)
    assert bool(torch.isfinite(out).all())
    near(out, *ex.forward()[:2], "out")


@pytest.mark.parametrize("shape", [(1, 40, 90, 2, 2, 64), (1, 3, 700, 4, 1, 72)])
@pytest.mark.parametrize("height", [10.0, -30.0])
def test_small_values(shape, height):
    q, k, v, _ = aligned_scores(shape, height)
    v = (v.float() * 2.0 ** -100).to(torch.bfloat16)
    ex = Exact(q, k, v)
    out, _ = T.attention(q, k, v)
    near(out, *ex.forward()[:2], "out")


@pytest.mark.parametrize("shape", [(1, 40, 90, 2, 2, 64), (2, 130, 700, 4, 2, 72)])
def test_gradients_of_large_values(shape):
    """Values of 2^60 and upstream gradients of 2^50: score gradients of 2^112."""
    q, k, v, do, _ = draw(*shape, torch.bfloat16)
    v, do = ((t.float() * 2.0 ** s).to(torch.bfloat16) for t, s in ((v, 60), (do, 50)))
    out, lse = T.attention(q, k, v, want_lse=True)
    got = T.attention_backward(do, q, k, v, out, lse)
    for g, r, t, name in zip(got, *Exact(q, k, v).backward(do, out, lse), ("dq", "dk", "dv")):
        assert bool(torch.isfinite(g).all()), name
        near(g, r, t, name)
