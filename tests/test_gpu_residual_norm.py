"""The residual stream's norm and its gradient against their formulas in 64 bits.

Tolerances: a result is rounded once to its type (half a step), and the fp32 work
before it is off by at most K half steps of 2^-24 of the formula's value with every
term taken as its absolute value.  K counts the roundings on the longest path: a
sum over a row adds at most 32 channels of a lane, six lane exchanges and 16 waves
(54), the mean enters the deviation and both enter the result (108), with fewer than
20 products and divisions between; through the branch's norm as well that is twice.
Sums over tokens add a group's rows, eight groups and the workgroups' parts.
"""
import math

import pytest
import torch

import paper_2608_03057_amd as T

pytestmark = pytest.mark.gpu

DEV = "cuda"
EPS = 1e-6
F32 = 2.0 ** -24
HALF = {torch.float32: F32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
K = 260


class Norm:
    """N of rows v in 64 bits, with the absolute form of its value and of its
    Jacobian's product."""

    def __init__(self, v, layer, eps):
        self.layer = layer
        mean = v.mean(-1, keepdim=True) if layer else torch.zeros_like(v[..., :1])
        c = v - mean
        self.d = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
        self.n = c * self.d
        # |v| + mean|v|, and what an error of the deviation is of the value
        self.abs = (v.abs() + (v.abs().mean(-1, keepdim=True) if layer else 0)) * self.d
        self.abs = self.abs * (1 + (self.abs ** 2).mean(-1, keepdim=True))

    def back(self, g):
        m = g.mean(-1, keepdim=True) if self.layer else 0
        return (g - m - self.n * (g * self.n).mean(-1, keepdim=True)) * self.d

    def back_abs(self, g):
        m = g.mean(-1, keepdim=True) if self.layer else 0
        inner = (g * self.abs).mean(-1, keepdim=True)
        return (g + m + self.abs * inner * (1 + (self.abs ** 2).mean(-1, keepdim=True))) * self.d

    def through(self, e):
        """What an error e of v is in n."""
        return self.back_abs(e)


def mod(t, fill, like):
    if t is None:
        return torch.full_like(like[:1, :1], fill)
    return t.double()[None, None] if t.dim() == 1 else t.double()[:, None]


def oracle_forward(x, y, gate, weight, scale, shift, post, layer, alpha, eps):
    """((r, its error), (h, its error)) without the last rounding, in units of
    2^-24."""
    x = x.double()
    r, er = x, torch.zeros_like(x)
    if y is not None:
        p, ep = y.double(), torch.zeros_like(x)
        if post is not None:
            n = Norm(p, layer, eps)
            p, ep = n.n * post.double(), K * n.abs * post.double().abs()
        g = mod(gate, 1.0, x)
        r = alpha * x + g * p
        er = ep * g.abs() + 3 * ((alpha * x).abs() + (g * p).abs())
    n = Norm(r, layer, eps)
    f = mod(weight, 1.0, x) * (1 + mod(scale, 0.0, x))
    fa = mod(weight, 1.0, x).abs() * (1 + mod(scale, 0.0, x).abs())
    s = mod(shift, 0.0, x)
    h = n.n * f + s
    eh = (K * n.abs + n.through(er)) * fa + s.abs()
    return (r, er), (h, eh)


def oracle_backward(dh, dr, r, y, gate, weight, scale, shift, post, layer, alpha, eps):
    """[(gradient, its error)] in ResidualGrads' order, None where there is none."""
    dh, r = dh.double(), r.double()
    dr = torch.zeros_like(r) if dr is None else dr.double()
    n = Norm(r, layer, eps)
    w, sc = mod(weight, 1.0, r), mod(scale, 0.0, r)
    f, fa = w * (1 + sc), w.abs() * (1 + sc.abs())
    D = dr + n.back(dh * f)
    Da = dr.abs() + n.back_abs(dh.abs() * fa)
    a = alpha if y is not None else 1.0

    def total(v, like):
        if like is None:
            return None
        return v.sum((0, 1)) if like.dim() == 1 else v.sum(1)
    count = K + 60 + r.shape[0] * r.shape[1] / 8

    def pair(v, va, like):
        return None if like is None else (total(v, like), count * total(va, like))
    out = [(a * D, K * abs(a) * Da), None, None, pair(dh * n.n * (1 + sc),
                                                      dh.abs() * n.abs * (1 + sc.abs()), weight),
           pair(dh * n.n * w, dh.abs() * n.abs * w.abs(), scale), pair(dh, dh.abs(), shift), None]
    if y is not None:
        y = y.double()
        g = mod(gate, 1.0, r)
        wp = mod(post, 1.0, r)
        p, pa = y, y.abs()
        if post is not None:
            q = Norm(y, layer, eps)
            p, pa = q.n, q.abs
        ga = D * g * wp
        gaa = Da * g.abs() * wp.abs()
        out[1] = (ga, K * gaa) if post is None else (q.back(ga), 2 * K * q.back_abs(gaa))
        out[2] = pair(D * p * wp, 2 * Da * pa * wp.abs(), gate)
        out[6] = pair(D * p * g, 2 * Da * pa * g.abs(), post)
    return out


def close(got, ref, err, dtype, name):
    assert got.dtype == dtype and got.shape == ref.shape, name
    tol = HALF[dtype] * (ref.abs() + F32 * err) + F32 * err + TINY[dtype]
    off = (got.double() - ref).abs()
    assert bool((off <= tol).all()), (name, float((off / tol).max()))


def make(B, S, C, dtype, mods="entry", wide=False, branch=True, post=False, weight=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, t=dtype, f=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * f).to(t)
    mt = torch.float32 if wide else dtype
    m = normal(*((6, C) if mods == "shared" else (B, 6, C)), t=mt, f=0.3)
    three = [None] * 3 if mods == "none" else [m[..., i, :] for i in (2, 4, 3)]
    return dict(
        x=normal(B, S, C, f=2.0) + 0.5, y=normal(B, S, C) if branch else None,
        gate=three[0] if branch else None, scale=three[1], shift=three[2],
        weight=1 + 0.2 * normal(C, t=torch.float32) if weight else None,
        post=1 + 0.2 * normal(C, t=torch.float32) if branch and post else None,
        dh=normal(B, S, C), dr=normal(B, S, C))


def check(a, kind="layer", alpha=1.0, eps=EPS, grad=True):
    layer, dtype = kind == "layer", a["x"].dtype
    how = dict(weight=a["weight"], scale=a["scale"], shift=a["shift"], post_weight=a["post"],
               kind=kind, residual_scale=alpha, eps=eps)
    ref = (a["y"], a["gate"], a["weight"], a["scale"], a["shift"], a["post"], layer, alpha, eps)
    r, h = T.residual_norm(a["x"], a["y"], a["gate"], **how)
    (rr, er), (rh, eh) = oracle_forward(a["x"], *ref)
    close(r, rr, er, dtype, "r")
    close(h, rh, eh, dtype, "h")
    if not grad:
        return
    got = T.residual_norm_backward(a["dh"], a["dr"], r, a["y"], a["gate"], **how)
    want = oracle_backward(a["dh"], a["dr"], r, *ref)
    for name, g, w in zip(got._fields, got, want):
        assert (g is None) == (w is None), name
        if g is not None:
            close(g, *w, dtype if name in ("dx", "dy") else torch.float32, name)


WIDTHS = [1, 2, 7, 8, 9, 63, 72, 500, 512, 513, 641, 1024, 1030, 1152, 1153, 1536, 1540, 2041,
          2048, 2240, 4096, 4099, 8192, 8200, 16383, 16384]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", list(HALF))
def test_widths(C, dtype):
    # (a row of one channel has no deviation: eps is all that its norm is made of)
    kind = "rms" if C == 1 else "layer"
    check(make(3, 11, C, dtype, weight=True, seed=C), kind)
    check(make(2, 5, C, dtype, mods="shared", wide=True, post=True, weight=C % 2 == 0, seed=C + 1),
          "rms", 0.5)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("mods", ["entry", "shared", "none"])
@pytest.mark.parametrize("branch,post", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("C,dtype", [(1152, torch.bfloat16), (77, torch.float32),
                                     (2240, torch.float16)])
def test_forms(kind, mods, branch, post, weight, C, dtype):
    check(make(2, 9, C, dtype, mods, mods == "entry", branch, post, weight), kind,
          0.7 if branch else 1.0)


@pytest.mark.parametrize("B,S", [(1, 1), (1, 7), (1, 4096), (64, 1), (5, 33), (3, 1000), (300, 3)])
@pytest.mark.parametrize("C", [72, 1152, 2241])
def test_tokens(B, S, C):
    check(make(B, S, C, torch.bfloat16, weight=True, post=C == 72))


@pytest.mark.parametrize("layer_eps", [0.0, 1e-5, 1.0])
def test_eps(layer_eps):
    check(make(2, 6, 200, torch.float32), "layer", eps=layer_eps)
    check(make(2, 6, 200, torch.float32, post=True), "rms", eps=layer_eps)


def test_negative_and_zero_scale():
    check(make(2, 6, 200, torch.float32), alpha=-1.5)
    check(make(2, 6, 200, torch.float32), alpha=0.0)


@pytest.mark.parametrize("C", [1152, 645])
def test_strides(C):
    """Operands as slices of wider rows, tokens outermost, entries expanded."""
    a = make(4, 6, C, torch.bfloat16, wide=True, post=True, weight=True)
    plain = {n: None if t is None else t.clone() for n, t in a.items()}
    g = torch.Generator(device=DEV).manual_seed(9)
    wide = torch.randn(4, 6, 3, C + 5, generator=g, device=DEV).bfloat16()
    for i, n in enumerate(("x", "y", "dh")):
        wide[:, :, i, 3:3 + C] = a[n]
        a[n] = wide[:, :, i, 3:3 + C]
    turned = torch.empty(6, 4, C, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    turned.copy_(a["dr"])
    a["dr"] = turned
    a["gate"] = a["gate"][:1].expand(4, C)
    plain["gate"] = a["gate"].contiguous()
    how = [dict(weight=d["weight"], scale=d["scale"], shift=d["shift"], post_weight=d["post"])
           for d in (a, plain)]
    one, two = (T.residual_norm(d["x"], d["y"], d["gate"], **k) for d, k in zip((a, plain), how))
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    grads = [T.residual_norm_backward(d["dh"], d["dr"], one[0], d["y"], d["gate"], **k)
             for d, k in zip((a, plain), how)]
    assert all(torch.equal(p, q) for p, q in zip(*grads))
    assert grads[0].dgate.shape == (4, C)           # of every entry, though one was given
    check(a)


def test_in_place_residual():
    a = make(2, 9, 1152, torch.bfloat16)
    how = dict(scale=a["scale"], shift=a["shift"])
    r, h = T.residual_norm(a["x"], a["y"], a["gate"], **how)
    out = torch.empty_like(h)
    r2, h2 = T.residual_norm(a["x"], a["y"], a["gate"], **how, out_r=a["x"], out_h=out)
    assert r2 is a["x"] and h2 is out and torch.equal(r2, r) and torch.equal(h2, h)


def test_without_branch_the_stream_is_returned():
    a = make(2, 9, 640, torch.float16, branch=False)
    r, _ = T.residual_norm(a["x"], scale=a["scale"])
    assert r is a["x"]


def test_no_later_use_of_r():
    a = make(2, 9, 640, torch.float32)
    a["dr"] = None
    check(a)


@pytest.mark.parametrize("B,S", [(0, 5), (2, 0)])
def test_nothing(B, S):
    a = make(B, S, 40, torch.bfloat16, weight=True, post=True)
    how = dict(weight=a["weight"], scale=a["scale"], shift=a["shift"], post_weight=a["post"])
    r, h = T.residual_norm(a["x"], a["y"], a["gate"], **how)
    assert r.shape == h.shape == (B, S, 40)
    g = T.residual_norm_backward(a["dh"], a["dr"], r, a["y"], a["gate"], **how)
    assert g.dx.shape == (B, S, 40) and g.dgate.shape == (B, 40)
    for t in (g.dgate, g.dscale, g.dshift, g.dweight, g.dpost_weight):
        assert not t.any()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("C", [96, 1160, 3001])
def test_values_that_are_not_finite_stay_in_their_row(bad, C):
    a = make(2, 8, C, torch.bfloat16)
    how = dict(scale=a["scale"], shift=a["shift"])
    r, h = T.residual_norm(a["x"], a["y"], a["gate"], **how)
    a["x"][1, 3, C // 2] = bad
    r2, h2 = T.residual_norm(a["x"], a["y"], a["gate"], **how)
    keep = torch.ones(2, 8, dtype=torch.bool, device=DEV)
    keep[1, 3] = False
    assert torch.equal(r2[keep], r[keep]) and torch.equal(h2[keep], h[keep])
    assert not torch.isfinite(h2[1, 3]).any()


def test_rows_far_apart():
    """Offsets past 2^31 elements and 2^32 bytes."""
    C, far = 520, (1 << 31) + 40
    flat = torch.empty(2 * far + C, dtype=torch.bfloat16, device=DEV)
    a = make(1, 3, C, torch.bfloat16)
    for n in ("x", "dh"):
        t = flat.as_strided((1, 3, C), (0, far, 1))
        t.copy_(a[n])
        a[n] = t
        check(a)
        a[n] = a[n].clone()


def test_many_tokens():
    """More than 2^31 elements of a stream, whose last rows are as they should be."""
    S, C = 140000, 16384
    x = torch.empty(1, S, C, dtype=torch.bfloat16, device=DEV)
    x[:, :-4] = 1.0
    x[:, -4:] = make(1, 4, C, torch.bfloat16)["x"]
    _, h = T.residual_norm(x, kind="rms")
    a = dict.fromkeys(("y", "gate", "weight", "scale", "shift", "post"))
    _, (rh, eh) = oracle_forward(x[:, -4:], *a.values(), False, 1.0, EPS)
    close(h[:, -4:].clone(), rh, eh, torch.bfloat16, "h")
    dh = h
    g = T.residual_norm_backward(dh, None, x, kind="rms")
    (dx, e), *_ = oracle_backward(h[:, -4:], None, x[:, -4:], *a.values(), False, 1.0, EPS)
    close(g.dx[:, -4:].clone(), dx, e, torch.bfloat16, "dx")


def test_same_bits_each_time():
    a = make(3, 1000, 1152, torch.bfloat16, weight=True, post=True)
    how = dict(weight=a["weight"], scale=a["scale"], shift=a["shift"], post_weight=a["post"])
    runs = [T.residual_norm_backward(a["dh"], a["dr"], a["x"], a["y"], a["gate"], **how)
            for _ in range(3)]
    for other in runs[1:]:
        assert all(torch.equal(p, q) for p, q in zip(runs[0], other))


def test_captured_and_replayed():
    a = make(2, 300, 1152, torch.bfloat16, weight=True)
    how = dict(weight=a["weight"], scale=a["scale"], shift=a["shift"])

    def both():
        r, h = T.residual_norm(a["x"], a["y"], a["gate"], **how)
        return (r, h, *T.residual_norm_backward(a["dh"], a["dr"], r, a["y"], a["gate"], **how)[:6])
    both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(3):
        b = make(2, 300, 1152, torch.bfloat16, weight=True, seed=seed + 5)
        for n in ("x", "y", "dh", "dr"):
            a[n].copy_(b[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, both()))


@pytest.mark.parametrize("kind,post", [("layer", False), ("rms", True), ("layer", True)])
def test_gradient_against_differences(kind, post):
    """The change of L = sum(h ch + r cr) along a direction, by central differences of
    the forward kernel at steps s and s/2, against the gradients' product with it.
    The difference at s/2 is off by a third of what it moved (its error goes with
    s^2; three times that allowed), and by the rounding of the 2 n terms of L."""
    a = make(2, 5, 130, torch.float32, wide=True, weight=True, post=post, seed=3)
    names = ("x", "y", "gate", "weight", "scale", "shift", "post")
    alpha = 0.8
    g = torch.Generator(device=DEV).manual_seed(4)
    a["gate"], a["scale"], a["shift"] = (a[n].clone() for n in ("gate", "scale", "shift"))

    def run(d):
        return T.residual_norm(d["x"], d["y"], d["gate"], weight=d["weight"], scale=d["scale"],
                               shift=d["shift"], post_weight=d["post"], kind=kind,
                               residual_scale=alpha)
    r, _ = run(a)
    grads = T.residual_norm_backward(a["dh"], a["dr"], r, a["y"], a["gate"], weight=a["weight"],
                                     scale=a["scale"], shift=a["shift"], post_weight=a["post"],
                                     kind=kind, residual_scale=alpha)
    of = dict(x=grads.dx, y=grads.dy, gate=grads.dgate, weight=grads.dweight, scale=grads.dscale,
              shift=grads.dshift, post=grads.dpost_weight)
    for n in names:
        if a[n] is None:
            continue
        way = torch.randn(a[n].shape, generator=g, device=DEV)

        def value(step):
            r, h = run({**a, n: a[n] + step * way})
            terms = (r.double() * a["dr"].double(), h.double() * a["dh"].double())
            return sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
        slopes, size = [], 0.0
        for s in (2.0 ** -6, 2.0 ** -7):
            (up, size), (down, _) = value(s), value(-s)
            slopes.append((up - down) / (2 * s))
        rounding = K * F32 * size / 2.0 ** -7
        want = float((of[n].double() * way.double()).sum())
        slack = abs(slopes[0] - slopes[1]) + rounding
        assert abs(slopes[1] - want) <= slack, (n, slopes, want, slack)
