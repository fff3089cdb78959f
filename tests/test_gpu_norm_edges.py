"""Norm and rotation of heads where sizes or values end: no eps, heads that are no
multiple of the four that a group of lanes takes.  Bounds as in
test_gpu_norm_rotate."""
import pytest
import torch

import paper_2608_03057_amd as T
from test_gpu_norm_rotate import backward, forward, near, tables

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("dim,rot,inter", [(64, 64, False), (64, 64, True), (72, 36, False),
                                           (40, 0, False), (136, 136, False), (70, 34, False)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_eps(heads, dim, rot, inter, dtype):
    g = torch.Generator().manual_seed(heads + dim)
    q = torch.randn(2, 9, heads, dim, generator=g).to(dtype).to(DEV)
    k = torch.randn(2, 5, 3, dim, generator=g).to(dtype).to(DEV)
    dq, dk = (torch.randn(t.shape, generator=g).to(dtype).to(DEV) for t in (q, k))
    wq, wk = (torch.randn(dim, generator=g).to(DEV) for _ in range(2))
    rope = (*tables(9, rot), None) if rot else None
    yq, yk = T.qk_norm_rotate(q, k, wq, wk, rope, rope, eps=0.0, interleaved=inter)
    near(yq, *forward(q, wq, rope, inter, 0.0), 24)
    near(yk, *forward(k, wk, rope, inter, 0.0), 24)
    gq, gk, dwq, dwk = T.qk_norm_rotate_backward(dq, dk, q, k, wq, wk, rope, rope, eps=0.0,
                                                 interleaved=inter)
    for got, dw, d, x, w in ((gq, dwq, dq, q, wq), (gk, dwk, dk, k, wk)):
        dx, mag, rw, wmag = backward(d, x, w, rope, inter, 0.0)
        near(got, dx, mag, 48)
        near(dw, rw, wmag, 24 + x.numel() / dim / 256 + 64)
