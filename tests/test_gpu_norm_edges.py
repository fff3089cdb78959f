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


def test_no_gradient_of_keys_that_are_none():
    """Keys of no token need no gradient; their weight's is zeros, not what the
    memory held."""
    g = torch.Generator().manual_seed(1)
    q = torch.randn(1, 5, 3, 64, generator=g).to(DEV)
    w = torch.ones(64, device=DEV)
    full = [torch.full((64,), 7.0, device=DEV) for _ in range(64)]
    del full                                # the memory that is allocated next
    _, gk, _, dwk = T.qk_norm_rotate_backward(q, None, q, q[:, :0], w, w)
    assert gk.shape == (1, 0, 3, 64) and torch.equal(dwk, torch.zeros_like(w))
    with pytest.raises(T.TasqError):        # keys that need one
        T.qk_norm_rotate_backward(q, None, q, q, w, w)


def test_more_workgroups_than_a_launch_takes():
    """2^24 groups of eight heads of 136 and some: tokens one element apart, 36 GB out."""
    torch.cuda.empty_cache()
    S, D = (1 << 27) + 5000, 136
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    g = torch.Generator(device=DEV).manual_seed(2)
    buf = torch.randn(S + D, generator=g, device=DEV).to(torch.bfloat16)
    x = torch.as_strided(buf, (1, S, 1, D), (0, 1, 0, 1))
    w = torch.randn(D, generator=g, device=DEV)
    k = torch.randn(1, 9, 3, D, generator=g, device=DEV).to(torch.bfloat16)
    y = torch.full((1, S, 1, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    _, yk = T.qk_norm_rotate(x, k, w, w, out_q=y)
    torch.cuda.synchronize()
    near(yk, *forward(k, w, None, False), 24)
    for first in [i * (1 << 25) - 3000 for i in range(1, 5)] + [0, S - 6000]:
        at = slice(first, first + 6000)
        near(y[:, at], *forward(x[:, at], w, None, False), 24)
    for first in range(0, S, 1 << 24):
        assert not bool(y[:, first:first + (1 << 24)].isnan().any())
    del y
    torch.cuda.empty_cache()
