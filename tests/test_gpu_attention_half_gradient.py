"""Attention's gradient in half where the score gradients ds leave half's range:
upstream gradients of any size, long rows, rows of different sizes.

The kernels scale the ds by a power of two: that of a query (for dq) follows its
upstream gradients, that of a key (for dk) those of the first queries, to a
largest of 2^8, with a factor of 2^14 at most; a column whose sums pass half's
range all the same is computed again with a factor lower by 2^15, so that its
largest ds is above 2.  A ds is then off by U of itself, or by the half step 2^-25
of the scaled values where it is below the normal numbers: by 2^-33 of the
upstream gradients' largest (2^-39 at least), or by 2^-26 of the largest ds, as it
is computed.  So, with a, e and U as in test_gpu_attention,
  |dq - ref| <= scale sum_j (U |ds| + 2 e a + step) |k| + U |ref| + 2^-25,
  step = max(2^-33 max(2^-6, |do|), 2^-26 max (|ds| + 2 e a)),
the maxima over the query (for dq) and over all queries (for dk).
Those bounds add up magnitudes; the roundings are independent, so the
error's norm is far below them.  Of independent roundings of U each, uniform, of ds
and of the result the error is sqrt(2 / 3) U of the norm where terms do not
cancel more than random signs do, and 2^-25 / sqrt(3) an element of a result
below the normal numbers: asserted are 2 U of the norm and 2^-25 an element."""
import math

import pytest
import torch

import paper_2608_03057_amd as T
from test_gpu_attention import Exact, U, bmm, draw, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = torch.float16
STEP = 2.0 ** -25


def bounds(ex, do, out, lse):
    """(reference, bound) of dq, dk and dv."""
    refs, _ = ex.backward(do, out, lse)
    do, out = do.double().transpose(1, 2), out.double().transpose(1, 2)
    p = ex.weights(lse.double())
    inner = (do * out).sum(-1, keepdim=True)
    ds = p * (bmm(do, ex.v.transpose(2, 3)) - inner)
    a = p * (bmm(do.abs(), ex.v.abs().transpose(2, 3)) + (do * out).abs().sum(-1, keepdim=True))
    size = ds.abs() + 2 * ex.e * a
    u, live = U[HALF], ex.live.double()
    each = u * ds.abs() + 2 * ex.e * a
    low, high = 2.0 ** -33, 2.0 ** -26
    top = do.abs().clamp(min=2.0 ** -6)
    row = (each + live * torch.maximum(low * top.amax(3, keepdim=True),
                                       high * size.amax(3, keepdim=True))) * ex.scale
    key = (each + live * torch.maximum(low * top.amax(),
                                       high * size.amax(2, keepdim=True))) * ex.scale

    def shared(t):
        B, H, S, D = t.shape
        return t.reshape(B, ex.HK, ex.G, S, D).sum(2).transpose(1, 2)
    tols = [bmm(row, ex.k.abs()).transpose(1, 2),
            shared(bmm(key.transpose(2, 3), ex.q.abs())),
            shared(bmm(((u + ex.e) * p + STEP * live).transpose(2, 3), do.abs()))]
    return [(r, t + u * r.abs() + STEP) for r, t in zip(refs, tols)]


def check(q, k, v, do, lengths=None, mask=None, norms=True, workspace=None):
    ex = Exact(q, k, v, lengths, mask)
    out, lse = T.attention(q, k, v, kv_lengths=lengths, key_mask=mask, want_lse=True)
    got = T.attention_backward(do, q, k, v, out, lse, kv_lengths=lengths, key_mask=mask,
                               workspace=workspace)
    for g, (ref, tol), name in zip(got, bounds(ex, do, out, lse), ("dq", "dk", "dv")):
        assert bool(torch.isfinite(g).all()), name
        near(g, ref, tol, name)
        if norms:
            room = 2 * U[HALF] * float(ref.norm()) + STEP * math.sqrt(ref.numel())
            assert float((g.double() - ref).norm()) <= room, (name, float(ref.norm()))


SHAPES = [(1, 512, 4096, 1, 1, 64), (2, 130, 1500, 4, 2, 72), (1, 700, 600, 2, 1, 128),
          (1, 1, 3000, 4, 1, 80), (1, 3000, 65, 2, 2, 40)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("size", [0, -10, -16])
def test_small_upstream_gradients(shape, size):
    q, k, v, do, _ = draw(*shape, HALF)
    check(q, k, v, (do.float() * 2.0 ** size).half())


@pytest.mark.parametrize("shape", SHAPES[:3])
def test_one_range(shape):
    q, k, v, do, _ = draw(*shape, HALF)
    rows = torch.empty((4 * shape[0] * shape[1] * shape[3] + 255) // 256 * 256,
                       dtype=torch.uint8, device=DEV)
    check(q, k, v, (do.float() * 2.0 ** -12).half(), workspace=rows)


@pytest.mark.parametrize("shape", [(1, 40, 9, 2, 2, 64), (2, 130, 70, 4, 2, 72)])
def test_large_upstream_gradients(shape):
    """Score gradients past 65504 whose products with small q and k are not."""
    q, k, v, do, _ = draw(*shape, HALF)
    q, k = (q.float() * 2.0 ** -7).half(), (k.float() * 2.0 ** -7).half()
    v, do = (v.float() * 2.0 ** 6).half(), (do.float() * 2.0 ** 12).half()
    ex = Exact(q, k, v)
    out, lse = T.attention(q, k, v, want_lse=True)
    dp = bmm(do.double().transpose(1, 2), ex.v.transpose(2, 3))
    inner = (do.double() * out.double()).sum(-1).transpose(1, 2)[..., None]
    assert float((ex.weights(lse.double()) * (dp - inner)).abs().max()) > 65504
    check(q, k, v, do)


@pytest.mark.parametrize("shape", [(1, 300, 1100, 2, 2, 64), (2, 200, 700, 4, 1, 72)])
def test_rows_of_all_sizes(shape):
    """Upstream gradients from 2^-20 to 2^3 from query to query, rows of zeros
    among them, and scores that rise along the keys."""
    q, k, v, do, g = draw(*shape, HALF)
    B, SQ, SK = shape[:3]
    size = torch.randint(-20, 4, (B, SQ, 1, 1), generator=g).float()
    do = (do.float() * torch.exp2(size).to(DEV)).half()
    do[:, ::7] = 0.0
    check(q, k, v, do, norms=False)
    ramp = torch.linspace(0.05, 3.0, SK, device=DEV)[None, :, None, None]
    check(q, (k.float() * ramp).half(), v, do, norms=False)
    check(q, (k.float() * ramp.flip(1)).half(), v, do, norms=False)


def test_small_gradients_with_masks_and_lengths():
    shape = (3, 140, 500, 4, 2, 64)
    q, k, v, do, g = draw(*shape, HALF)
    do = (do.float() * 2.0 ** -14).half()
    mask = (torch.rand(3, 500, generator=g) < 0.5).to(DEV)
    mask[0, :130] = False
    mask[1, 1:] = False
    mask[1, 0] = True
    lengths = torch.tensor([500, 300, 65], dtype=torch.int32, device=DEV)
    kk = torch.where(mask[:, :, None, None], k, math.nan)
    vv = torch.where(mask[:, :, None, None], v, math.inf)
    check(q, kk, vv, do, mask=mask, norms=False)
    check(q, kk, vv, do, mask=mask, lengths=lengths, norms=False)


def test_a_broken_row_stays_in_its_query():
    """A NaN upstream gradient: dq of the other queries keeps its bits."""
    q, k, v, do, _ = draw(1, 70, 200, 2, 2, 64, HALF)
    out, lse = T.attention(q, k, v, want_lse=True)
    clean = T.attention_backward(do, q, k, v, out, lse)[0]
    do[0, 9, 1, 5] = math.nan
    got = T.attention_backward(do, q, k, v, out, lse)[0]
    assert bool(got[0, 9, 1].isnan().all())
    keep = torch.ones(70, 2, dtype=torch.bool, device=DEV)
    keep[9, 1] = False
    assert torch.equal(got[0][keep], clean[0][keep])


@pytest.mark.parametrize("shape", [(1, 300, 200, 2, 2, 64), (2, 150, 90, 4, 2, 128)])
def test_upstream_gradients_that_grow_along_the_queries(shape):
    """The first tile of queries says nothing of the others: up to 2^20 times as
    large, against the largest values that dq, dk and dv have room for."""
    q, k, v, do, _ = draw(*shape, HALF)
    SQ = shape[1]
    size = torch.where(torch.arange(SQ) < 64, -16.0, 4.0)
    do = (do.float() * torch.exp2(size).to(DEV)[None, :, None, None]).half()
    k, v = (k.float() * 4).half(), (v.float() * 16).half()
    check(q, k, v, do, norms=False)
    check(q, k, v, do.flip(1), norms=False)
