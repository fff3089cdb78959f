"""Norm and rotation of heads, and their gradient, against the formulas in 64
bits.

Forward bound: the sum of dim squares is a chain of at most 20 fp32
roundings, halved by the root; the root, the mean, three products and the
rotation add ten more, so an element is within 24 * 2^-24 of
(|n1 c| + |n2 s|).  Backward: dx = r (g w - x t) with t a second such sum,
whose roundings are relative to mean |g w x|: 48 * 2^-24 of r (|g w| + |x| r^2
mean |g w x|).  dw is a sum of N terms, each 24 roundings off, added over
chains of at most (N / 256 + 64) terms: (24 + N / 256 + 64) * 2^-24 of the sum
of magnitudes.  16-bit results add half a unit in the last place."""
import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -140, torch.bfloat16: 2.0 ** -130, torch.float16: 2.0 ** -25}
EPS = 1e-6


def tables(P, rot, seed=0):
    g = torch.Generator().manual_seed(seed)
    ang = 20 * torch.rand(P, rot // 2, generator=g)
    return torch.cos(ang).to(DEV), torch.sin(ang).to(DEV)


def turn(x, rope, interleaved, back=False):
    """Rotation in 64 bits and the magnitudes of its terms; x [B, S, H, D]."""
    y, mag = x.clone(), x.abs()
    if rope is None:
        return y, mag
    cos, sin, pos = rope
    B, S, H, D = x.shape
    half = cos.shape[1]
    pos = torch.arange(S, device=x.device).expand(B, S) if pos is None else pos.long()
    inside = (pos >= 0) & (pos < cos.shape[0])
    c, s = (t.double()[pos.clamp(0, cos.shape[0] - 1)] for t in (cos, sin))
    c = torch.where(inside[..., None], c, torch.ones_like(c))[:, :, None]
    s = torch.where(inside[..., None], s, torch.zeros_like(s))[:, :, None]
    s = -s if back else s
    i = torch.arange(half, device=x.device)
    i, j = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    mag[..., i], mag[..., j] = ((x[..., i] * c).abs() + (x[..., j] * s).abs(),
                                (x[..., i] * s).abs() + (x[..., j] * c).abs())
    return y, mag


def forward(x, w, rope, interleaved, eps=EPS):
    x = x.double()
    r = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    return turn(x * r * (1.0 if w is None else w.double()), rope, interleaved)


def backward(dy, x, w, rope, interleaved, eps=EPS):
    """dx, its magnitudes, dw, its magnitudes."""
    dt, x = dy.dtype, x.double()
    g, gm = turn(dy.double(), rope, interleaved, back=True)
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    r = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    t = (g * w * x).mean(-1, keepdim=True) * r ** 2
    tm = (gm * w.abs() * x.abs()).mean(-1, keepdim=True) * r ** 2
    del dt
    return (r * (g * w - x * t), r * (gm * w.abs() + x.abs() * tm),
            (g * x * r).sum((0, 1, 2)), (gm * x.abs() * r).sum((0, 1, 2)))


def near(got, ref, mag, factor):
    dt = got.dtype
    tol = factor * U * mag + ROUND[dt] * ref.abs() * (1 + 2.0 ** -9) + TINY[dt]
    err = (got.double() - ref).abs()
    assert got.shape == ref.shape
    assert bool((err <= tol).all()), float((err - tol).max())


CASES = [
    # B, S, H, HK, D, rot, interleaved, positions
    (1, 1, 16, 16, 72, 72, False, False), (2, 37, 16, 16, 72, 72, False, True),
    (2, 19, 20, 5, 112, 112, True, False), (1, 65, 10, 10, 64, 32, False, True),
    (3, 7, 3, 1, 128, 64, True, True), (2, 5, 7, 2, 40, 40, False, False),
    (1, 9, 4, 4, 32, 0, False, False), (2, 3, 5, 1, 256, 128, False, True),
    (1, 11, 2, 1, 136, 136, True, False),
    # no whole groups of eight: any even size
    (2, 5, 3, 3, 2, 2, False, False), (1, 4, 5, 2, 70, 34, False, True),
    (1, 4, 5, 2, 70, 34, True, True), (2, 3, 2, 1, 250, 250, False, False),
    (2, 3, 2, 1, 36, 4, True, False),
]


def inputs_of(case, dtype, seed=0):
    B, S, H, HK, D, rot, inter, positions = case
    g = torch.Generator().manual_seed(seed + S * 100 + D)
    qkv = torch.randn(B, S, H + 2 * HK, D, generator=g).mul(2.0).to(dtype).to(DEV)
    q, k = qkv[:, :, :H], qkv[:, :, H:H + HK]
    wq, wk = (torch.randn(D, generator=g).to(DEV) for _ in range(2))
    rope = None
    if rot:
        pos = None
        if positions:               # some of them outside the table
            pos = torch.randint(-3, S + 3, (B, S), generator=g, dtype=torch.int32).to(DEV)
        rope = (*tables(S, rot), pos)
    return q, k, wq, wk, rope, inter, g


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_forward(case, dtype):
    q, k, wq, wk, rope, inter, _ = inputs_of(case, dtype)
    yq, yk = T.qk_norm_rotate(q, k, wq, wk, rope, rope, eps=EPS, interleaved=inter)
    near(yq, *forward(q, wq, rope, inter), 24)
    near(yk, *forward(k, wk, rope, inter), 24)


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_backward(case, dtype):
    q, k, wq, wk, rope, inter, g = inputs_of(case, dtype)
    dq, dk = (torch.randn(t.shape, generator=g).to(dtype).to(DEV) for t in (q, k))
    gq, gk, dwq, dwk = T.qk_norm_rotate_backward(dq, dk, q, k, wq, wk, rope, rope, eps=EPS,
                                                 interleaved=inter)
    for got, dw, d, x, w in ((gq, dwq, dq, q, wq), (gk, dwk, dk, k, wk)):
        dx, mag, rw, wmag = backward(d, x, w, rope, inter)
        near(got, dx, mag, 48)
        terms = x.numel() // x.shape[-1]
        near(dw, rw, wmag, 24 + terms / 256 + 64)


def test_gradient_against_differences():
    """Central differences of the 64-bit forward pass: truncation of order
    h^2, so 1e-6 of the gradient's size at h = 1e-4."""
    case = (1, 3, 2, 1, 24, 16, False, False)
    q, k, wq, wk, rope, inter, g = inputs_of(case, torch.float32)
    q = q.contiguous()
    dq = torch.randn(q.shape, generator=g).to(DEV)
    gq, _, dwq, _ = T.qk_norm_rotate_backward(dq, None, q, None, wq, None, rope, interleaved=inter)

    def loss(x, w):
        return float((forward(x, w, rope, inter)[0] * dq.double()).sum())
    h = 1e-4
    for where, grad, make in (
            (q, gq, lambda e: (q.double() + e, wq)), (wq, dwq, lambda e: (q, wq.double() + e))):
        for i in range(0, where.numel(), 7):
            e = torch.zeros(where.numel(), dtype=torch.float64, device=DEV)
            e[i] = h
            e = e.view(where.shape)
            num = (loss(*make(e)) - loss(*make(-e))) / (2 * h)
            assert abs(num - float(grad.flatten()[i])) <= 1e-5 * float(grad.abs().max()) + 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_and_ragged(dtype):
    """More tokens than a launch holds at once, keys of another length, no
    rotation of the keys, and no weights."""
    g = torch.Generator().manual_seed(5)
    q = torch.randn(3, 2049, 6, 72, generator=g).to(dtype).to(DEV)
    k = torch.randn(3, 77, 2, 72, generator=g).to(dtype).to(DEV)
    rope = (*tables(2049, 72), None)
    yq, yk = T.qk_norm_rotate(q, k, None, None, rope, None)
    near(yq, *forward(q, None, rope, False), 24)
    near(yk, *forward(k, None, None, False), 24)
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    w = torch.ones(72, device=DEV)
    gq, gk, dwq, dwk = T.qk_norm_rotate_backward(dq, dk, q, k, w, None, rope, None)
    assert dwk is None
    dx, mag, rw, wmag = backward(dq, q, w, rope, False)
    near(gq, dx, mag, 48)
    near(dwq, rw, wmag, 24 + 3 * 2049 * 6 / 256 + 64)
    dx, mag, _, _ = backward(dk, k, None, None, False)
    near(gk, dx, mag, 48)
    again = T.qk_norm_rotate_backward(dq, dk, q, k, w, None, rope, None)
    assert torch.equal(again[2], dwq) and torch.equal(again[0], gq)


def test_strides_and_alignment():
    """Heads before tokens, a base off the vector alignment, broadcast heads."""
    g = torch.Generator().manual_seed(6)
    buf = torch.randn(2, 4, 33, 73, generator=g).to(torch.bfloat16).to(DEV)
    w = torch.randn(72, generator=g).to(DEV)
    rope = (*tables(33, 72), None)
    wide = torch.randn(2, 33, 1, 72, generator=g).to(torch.bfloat16).to(DEV).expand(2, 33, 3, 72)
    for x in (buf[..., :72].transpose(1, 2), buf[..., 1:].transpose(1, 2), wide):
        for inter in (False, True):
            y, _ = T.qk_norm_rotate(x, None, w, None, rope, interleaved=inter)
            near(y, *forward(x, w, rope, inter), 24)
            dx = T.qk_norm_rotate_backward(x, None, x, None, w, None, rope, interleaved=inter)[0]
            ref, mag, _, _ = backward(x, x, w, rope, inter)
            near(dx, ref, mag, 48)


def test_heads_of_zeros_and_huge_values():
    x = torch.zeros(1, 3, 2, 64, device=DEV)
    x[0, 1] = 1e15                          # its square is far from overflow
    y, _ = T.qk_norm_rotate(x, None)
    assert torch.equal(y[0, 0], torch.zeros(2, 64, device=DEV))
    near(y, *forward(x, None, None, False), 24)


def test_empty_tensors():
    w = torch.ones(64, device=DEV)
    q = torch.empty(2, 0, 4, 64, device=DEV)
    k = torch.randn(2, 3, 4, 64, device=DEV)
    yq, yk = T.qk_norm_rotate(q, k, w, w)
    near(yk, *forward(k, w, None, False), 24)
    gq, gk, dwq, dwk = T.qk_norm_rotate_backward(q, k, q, k, w, w)
    assert yq.shape == gq.shape == q.shape
    assert torch.equal(dwq, torch.zeros_like(w)) and float(dwk.abs().max()) > 0
    gq, _, dwq, _ = T.qk_norm_rotate_backward(q, None, q, None, w)
    assert torch.equal(dwq, torch.zeros_like(w))


def test_refusals_of_the_wrappers():
    q = torch.randn(1, 4, 2, 64, device=DEV)
    cos, sin = tables(4, 64)
    with pytest.raises(ValueError):
        T.qk_norm_rotate(q[0], None)
    with pytest.raises(ValueError):
        T.qk_norm_rotate(q, q.to(torch.bfloat16))
    with pytest.raises(ValueError):
        T.qk_norm_rotate(q.transpose(2, 3), None)
    with pytest.raises(ValueError):
        T.qk_norm_rotate(q, None, torch.ones(32, device=DEV))
    with pytest.raises(ValueError):
        T.qk_norm_rotate(q, None, None, None, (cos, sin, torch.zeros(1, 3, dtype=torch.int32,
                                                                     device=DEV)))
    with pytest.raises(T.TasqError):        # rotated elements past the head
        T.qk_norm_rotate(q, None, None, None, (*tables(4, 96), None))
    with pytest.raises(T.TasqError):        # an odd head dimension
        T.qk_norm_rotate(q[..., :63], None)
    with pytest.raises(T.TasqError):
        T.qk_norm_rotate(q, None, eps=-1.0)
    with pytest.raises(T.TasqError):
        T.qk_norm_rotate_backward(q, None, q, None,
                                  workspace=torch.empty(256, dtype=torch.uint8, device=DEV))


# Whole groups of eight elements whose rotated part ends inside a group.
PART_GROUPS = [
    (1, 37, 6, 3, 72, 36, False, True), (2, 9, 5, 1, 40, 20, False, False),
    (2, 9, 5, 1, 40, 20, True, False), (1, 5, 3, 1, 64, 2, False, True),
    (1, 5, 3, 1, 128, 126, False, True), (1, 3, 2, 2, 256, 250, False, True),
    (1, 3, 2, 2, 256, 250, True, True), (2, 3, 2, 1, 24, 12, False, False),
    (3, 70, 9, 4, 104, 52, False, True),
]


@pytest.mark.parametrize("case", PART_GROUPS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rotation_that_ends_inside_a_group(case, dtype):
    test_forward(case, dtype)
    test_backward(case, dtype)


def test_one_rotation_ends_inside_a_group_and_one_does_not():
    g = torch.Generator().manual_seed(8)
    q = torch.randn(2, 21, 5, 72, generator=g).to(torch.bfloat16).to(DEV)
    k = torch.randn(2, 21, 3, 72, generator=g).to(torch.bfloat16).to(DEV)
    ropes = (*tables(21, 72), None), (*tables(21, 36, 1), None)
    y = T.qk_norm_rotate(q, k, None, None, *ropes)
    d = T.qk_norm_rotate_backward(q, k, q, k, None, None, *ropes)
    for i, (x, rope) in enumerate(zip((q, k), ropes)):
        near(y[i], *forward(x, None, rope, False), 24)
        near(d[i], *backward(x, x, None, rope, False)[:2], 48)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inter", [False, True])
def test_tables_weights_and_outputs_at_any_element(dtype, inter):
    g = torch.Generator().manual_seed(9)

    def off(t):         # the same values, one element after an aligned base
        b = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        b[1:] = t.reshape(-1)
        return b[1:].view(t.shape)
    x = torch.randn(2, 11, 3, 64, generator=g).to(dtype).to(DEV)
    w = torch.randn(64, generator=g).to(DEV)
    cos, sin = tables(11, 64)
    rope = (cos, sin, None)
    want, _ = T.qk_norm_rotate(x, None, w, None, rope, interleaved=inter)
    out = off(torch.zeros_like(x))
    got, _ = T.qk_norm_rotate(off(x), None, off(w), None, (off(cos), off(sin), None),
                              interleaved=inter, out_q=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
