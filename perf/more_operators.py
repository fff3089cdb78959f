"""Workload cases of what stands around a block's quantized linears.

Three operators and the direction each runs in:

  norm       the residual stream takes a branch's output through its gate, then
             the norm of the stream with the next branch's scale and shift,
             forward or backward
  mx4        activations -> 4-bit floating-point codes with one scale per 32,
             times a weight in the same form
  gradient   of the 8-bit linear with one scale per token, read from the codes
             that its forward pass took

A case names sizes, types and layout.  ``prepare`` draws what a program has in
hand before the call (the stream, modulations as slices of one projection,
stored weights, codes kept from the forward pass); ``run`` makes one pass;
``exact`` is the operator's definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def norm(B, S, C, t, kind="layer", branch=True, post=False, mod="entry", weight=False, alpha=1.0,
         grad=False):
    return {"op": "norm", "B": B, "S": S, "C": C, "t": t, "kind": kind, "branch": branch,
            "post": post, "mod": mod, "weight": weight, "alpha": alpha, "grad": grad}


def mx4(M, K, N, x, y, bias=True):
    return {"op": "mx4", "M": M, "K": K, "N": N, "x": x, "y": y, "bias": bias}


def gradient(M, K, N, b, t):
    return {"op": "gradient", "M": M, "K": K, "N": N, "b": b, "t": t}


def listed():
    cases = {
        # the time embedding's token in the 1152-wide block: latency
        "norm one token": norm(1, 1, 1152, "bf16"),
        # two 1024 px images between the attention and the MLP of a block
        "norm image": norm(2, 4096, 1152, "bf16"),
        # a 2240-wide block with norms on both sides of its branches, 512 px
        "norm both sides": norm(4, 1024, 2240, "f16", "rms", post=True, weight=True, alpha=0.7),
        # calibration on two 1024 px images
        "norm image gradient": norm(2, 4096, 1152, "bf16", grad=True),
        # texts of odd width in full precision, one modulation for all of them
        "norm text gradient": norm(3, 77, 641, "f32", "rms", post=True, mod="shared", weight=True,
                                   grad=True),
        # one token through the 1152-wide block's projection: a weight stream
        "mx4 one token": mx4(1, 1152, 3456, "bf16", "bf16"),
        # a text of odd length into keys and values, odd width
        "mx4 text": mx4(237, 640, 1283, "f16", "f16"),
        # two 1024 px images through the 1152-wide block's MLP
        "mx4 image": mx4(8192, 1152, 4608, "bf16", "bf16"),
        # the 2240-wide block's gated MLP, full precision at both ends
        "mx4 wide": mx4(4096, 2240, 11200, "f32", "f32", bias=False),
        # a text's projection of odd size
        "gradient text": gradient(300, 640, 1283, 6, "f16"),
        # two 1024 px images in the 1152-wide block's fused q, k, v
        "gradient image": gradient(8192, 1152, 3456, 8, "bf16"),
        # the 2240-wide block's gated MLP at a late stage's bits
        "gradient wide": gradient(4096, 2240, 11200, 4, "bf16"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    while True:
        kind = rng.choice(("norm", "norm", "norm gradient", "norm gradient", "mx4", "mx4", "few",
                           "gradient", "gradient"))
        t = rng.choice(("bf16", "f16"))
        wide = rng.random() < 0.5       # a width of whole vectors, or any
        if kind.startswith("norm"):
            C = _spread(rng, 4, 700) * 8 if wide else _spread(rng, 32, 5600)
            branch = rng.random() < 0.75
            case = norm(rng.randint(1, 8), _spread(rng, 1, 4096), C, rng.choice(("f32", t, t)),
                        rng.choice(("layer", "rms")), branch, branch and rng.random() < 0.4,
                        rng.choice(("entry", "entry", "shared", "none")), rng.random() < 0.5,
                        rng.choice((1.0, 0.5)) if branch else 1.0, kind.endswith("gradient"))
        else:
            K = _spread(rng, 4, 350) * 16 if wide else _spread(rng, 64, 5600)
            N = _spread(rng, 4, 1400) * 8 if wide else _spread(rng, 32, 11200)
            if kind == "gradient":
                case = gradient(_spread(rng, 1, 8192), K, N, rng.randint(2, 8), t)
            else:
                case = mx4(rng.randint(1, 16) if kind == "few" else _spread(rng, 1, 8192), K, N,
                           rng.choice(("f32", "bf16", "f16")), rng.choice(("f32", "bf16", "f16")),
                           rng.random() < 0.5)
        most = [work(c) for c in listed() if c["op"] == case["op"]]
        if all(work(case)[n] <= max(w[n] for w in most) for n in ("flops", "bytes")):
            return case


def work(case):
    c = case
    if c["op"] == "norm":
        n = c["B"] * c["S"] * c["C"]
        passes = (6 if c["branch"] else 4) if c["grad"] else (4 if c["branch"] else 2)
        return {"bytes": passes * n * BYTES[c["t"]], "flops": 5 * passes * n}
    M, N, K = c["M"], c["N"], c["K"]
    if c["op"] == "mx4":
        return {"bytes": M * K * BYTES[c["x"]] + N * K * 17 // 32 + M * N * BYTES[c["y"]],
                "flops": 2 * M * N * K}
    return {"bytes": 2 * M * N + M * K + N * K + 2 * M * K + 2 * N * K, "flops": 4 * M * N * K}


# ------------------------------------------------------------------- inputs

def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = case
    s = {"case": c}
    if c["op"] == "norm":
        B, S, C, t = c["B"], c["S"], c["C"], TYPES[c["t"]]
        s["x"] = _normal(g, B, S, C, dtype=t, scale=2.0)
        s["y"] = _normal(g, B, S, C, dtype=t) if c["branch"] else None
        # gate, scale and shift are slices of one projection of the time embedding
        mods = _normal(g, 1 if c["mod"] == "shared" else B, 6, C, dtype=t, scale=0.3)
        if c["mod"] == "shared":
            mods = mods[0]
        at = [None if c["mod"] == "none" else mods[..., i, :] for i in (2, 4, 3)]
        s["gate"], s["scale"], s["shift"] = at if c["branch"] else [None, *at[1:]]
        s["weight"] = 1 + 0.2 * _normal(g, C) if c["weight"] else None
        s["post"] = 1 + 0.2 * _normal(g, C) if c["post"] else None
        if c["grad"]:
            s["dr"] = _normal(g, B, S, C, dtype=t, scale=0.1)
            s["dh"] = _normal(g, B, S, C, dtype=t, scale=0.1)
            s["r"] = _norm(s)[0]                        # kept from the forward pass
        return s
    M, N, K = c["M"], c["N"], c["K"]
    # token magnitudes differ by a factor of ten or more, as activations' do
    spread = torch.exp(0.7 * torch.randn(M, 1, generator=g, device="cuda"))
    if c["op"] == "mx4":
        s["x"] = (_normal(g, M, K) * spread).to(TYPES[c["x"]])
        s["wc"], s["ws"] = _stored(_normal(g, N, K) / math.sqrt(K))
        s["bias"] = _normal(g, N) if c["bias"] else None
        return s
    x = _normal(g, M, K) * spread
    s["sx"] = x.abs().amax(1) / 127.0
    s["codes"] = torch.round(x / s["sx"][:, None]).clamp(-127, 127).to(torch.int8)
    s["W"] = torch.clamp(torch.round(_normal(g, N, K, scale=32.0)), -128, 127).to(torch.int8)
    s["sw"] = 1e-3 + 4e-3 * torch.rand(N, generator=g, device="cuda")
    s["dy"] = _normal(g, M, N, dtype=TYPES[c["t"]], scale=0.1)
    return s


# --------------------------------------------------------------- plain forms

def _center(s, v):
    """(v without its mean where the kind asks for it, 1 / deviation)"""
    if s["case"]["kind"] == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v, torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)


def _rows(m):
    """A modulation [C] or [B, C] as fp32 that meets [B, S, C]."""
    return m.float() if m.dim() == 1 else m.float()[:, None]


def _factor(s):
    """weight (1 + scale), as it meets [B, S, C]."""
    f = torch.ones(s["case"]["C"], device="cuda")
    if s["weight"] is not None:
        f = f * s["weight"]
    return f if s["scale"] is None else f * (1 + _rows(s["scale"]))


def _branch(s, y):
    """(the branch's output as the gate takes it, its normed values, 1 / deviation)"""
    if s["post"] is None:
        return y, y, None
    v, d = _center(s, y)
    n = v * d
    return n * s["post"], n, d


def _norm(s):
    t = s["x"].dtype
    r = s["x"].float()
    if s["y"] is not None:
        p, _, _ = _branch(s, s["y"].float())
        r = s["case"]["alpha"] * r + (p if s["gate"] is None else p * _rows(s["gate"]))
    v, d = _center(s, r)
    h = v * d * _factor(s)
    if s["shift"] is not None:
        h = h + _rows(s["shift"])
    return r.to(t), h.to(t)


def _through(s, g, n, d):
    """Gradient of the normed values n, through the norm."""
    back = g - n * (g * n).mean(-1, keepdim=True)
    if s["case"]["kind"] == "layer":
        back = back - g.mean(-1, keepdim=True)
    return back * d


def _sum(m, v):
    """v [B, S, C] summed to the shape of modulation m."""
    return v.sum((0, 1)) if m.dim() == 1 else v.sum(1)


def _norm_gradient(s):
    t, dh = s["r"].dtype, s["dh"].float()
    v, d = _center(s, s["r"].float())
    n = v * d
    D = s["dr"].float() + _through(s, dh * _factor(s), n, d)
    out = [(s["case"]["alpha"] * D if s["y"] is not None else D).to(t)]
    if s["y"] is not None:
        p, ny, dev = _branch(s, s["y"].float())
        g = D if s["gate"] is None else D * _rows(s["gate"])
        out.append((g if s["post"] is None else _through(s, g * s["post"], ny, dev)).to(t))
        if s["gate"] is not None:
            out.append(_sum(s["gate"], D * p))
    w = torch.ones_like(dh[0, 0]) if s["weight"] is None else s["weight"]
    if s["weight"] is not None:
        out.append((dh * n if s["scale"] is None else dh * n * (1 + _rows(s["scale"]))).sum((0, 1)))
    if s["scale"] is not None:
        out.append(_sum(s["scale"], dh * n * w))
    if s["shift"] is not None:
        out.append(_sum(s["shift"], dh))
    if s["post"] is not None:
        out.append((g * ny).sum((0, 1)))
    return out


def _blocks(x):
    """[rows, K] as fp32 blocks of 32, [rows, K / 32, 32], K filled up to a
    multiple of 128 with zeros."""
    x = x.float()
    x = torch.cat((x, x.new_zeros(x.shape[0], -x.shape[1] % 128)), 1)
    return x.reshape(x.shape[0], -1, 32)


def _codes(x):
    """(values of 4-bit codes [rows, K / 32, 32], exponents [rows, K / 32, 1])"""
    x = _blocks(x)
    e = torch.clamp(torch.frexp(x.abs().amax(-1, keepdim=True))[1] - 3, -127, 127)
    v = torch.ldexp(x, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.clamp(torch.round(a / step) * step, max=6.0)
    return torch.where(v < 0, -q, q), e


def _stored(w):
    """Codes uint8 [N, K / 2], the even element in the low half, and scales
    uint8 [N, K / 32], exponents plus 127."""
    q, e = _codes(w)
    a = q.abs()
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, torch.full_like(a, 7)))
    code = (code + torch.where(q < 0, 8.0, 0.0)).to(torch.uint8).flatten(1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e[..., 0] + 127).to(torch.uint8)


def _values(codes, scales):
    """fp32 values [N, K] of what _stored gives."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(1).int()
    a = (code & 7).float()
    a = torch.where(a <= 4, a / 2, torch.where(a < 7, a - 2, torch.full_like(a, 6.0)))
    v = torch.where(code > 7, -a, a).reshape(codes.shape[0], -1, 32)
    return torch.ldexp(v, scales.int()[..., None] - 127).flatten(1)


def _mx4(s):
    q, e = _codes(s["x"])
    x = torch.ldexp(q, e).flatten(1)
    y = torch.matmul(x, _values(s["wc"], s["ws"]).t().contiguous())
    return (y if s["bias"] is None else y + s["bias"]).to(TYPES[s["case"]["y"]])


def _gradient(s):
    t, dy = s["dy"].dtype, s["dy"].float()
    step = 2 ** (8 - s["case"]["b"])
    w = torch.floor(s["W"].float() / step) * step * s["sw"][:, None]
    x = s["codes"].float() * s["sx"][:, None]
    return [torch.matmul(dy, w).to(t), torch.matmul(dy.t().contiguous(), x).to(t), dy.sum(0)]


# ----------------------------------------------------------------- one pass

def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2608_03057_amd as T
        if c["op"] == "mx4":
            codes, scales = T.quantize_mx4(s["x"])
            return T.linear_mx4(codes, scales, s["wc"], s["ws"], s["bias"],
                                out_dtype=TYPES[c["y"]])
        if c["op"] == "gradient":
            return list(T.masked_linear_tokens_backward(s["dy"], s["codes"], s["W"], s["sx"],
                                                        s["sw"], c["b"]))
        how = dict(weight=s["weight"], scale=s["scale"], shift=s["shift"], post_weight=s["post"],
                   kind=c["kind"], residual_scale=c["alpha"], eps=EPS)
        if c["grad"]:
            return [t for t in T.residual_norm_backward(s["dh"], s["dr"], s["r"], s["y"],
                                                        s["gate"], **how) if t is not None]
        return list(T.residual_norm(s["x"], s["y"], s["gate"], **how))
    if c["op"] == "mx4":
        return _mx4(s)
    if c["op"] == "gradient":
        return _gradient(s)
    return _norm_gradient(s) if c["grad"] else list(_norm(s))


# ------------------------------------------------------------ 64-bit oracle

class _Exact:
    """Norm of rows in 64 bits, and the Jacobian's product, from the sums of
    powers."""

    def __init__(self, s, v):
        self.C, self.layer = v.shape[-1], s["case"]["kind"] == "layer"
        mean = v.sum(-1, keepdim=True) / self.C if self.layer else 0.0
        self.dev = ((v ** 2).sum(-1, keepdim=True) / self.C - mean ** 2 + EPS) ** 0.5
        self.n = (v - mean) / self.dev

    def back(self, g):
        inner = torch.linalg.vecdot(g, self.n)[..., None] / self.C
        mean = g.sum(-1, keepdim=True) / self.C if self.layer else 0.0
        return (g - mean - self.n * inner) / self.dev


def _wide(s, name, fill):
    """A modulation or weight in 64 bits as [B or 1, 1, C]."""
    m = s[name]
    if m is None:
        return torch.full((1, 1, s["case"]["C"]), fill, dtype=torch.float64, device="cuda")
    return m.double().reshape(-1, 1, s["case"]["C"])


def _exact_norm(s):
    c = s["case"]
    gate, w, post = _wide(s, "gate", 1.0), _wide(s, "weight", 1.0), _wide(s, "post", 1.0)
    scale, shift = _wide(s, "scale", 0.0), _wide(s, "shift", 0.0)
    branch = after = None
    if s["y"] is not None:
        branch = s["y"].double()
        if c["post"]:
            after = _Exact(s, branch)
            branch = after.n * post
    if not c["grad"]:
        r = s["x"].double()
        if branch is not None:
            r = c["alpha"] * r + gate * branch
        return [r, _Exact(s, r).n * w * (1 + scale) + shift]
    dh, at = s["dh"].double(), _Exact(s, s["r"].double())
    D = s["dr"].double() + at.back(dh * w * (1 + scale))
    per_entry = c["mod"] == "entry"

    def total(v):                       # to a modulation's shape
        return v.sum(1) if per_entry else v.flatten(0, 1).sum(0)
    some = c["mod"] != "none"
    out = [D if branch is None else c["alpha"] * D]
    if branch is not None:
        out.append(after.back(D * gate * post) if c["post"] else D * gate)
        if some:
            out.append(total(D * branch))
    if c["weight"]:
        out.append((dh * at.n * (1 + scale)).flatten(0, 1).sum(0))
    if some:
        out += [total(dh * at.n * w), total(dh)]
    if c["post"]:
        out.append((D * gate * after.n).flatten(0, 1).sum(0))
    return out


GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_mx4(s):
    # The codes are decisions on exact quotients: a value goes up a step of the
    # grid past the middle of it, and in the middle to the even place.
    c = s["case"]
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")

    def values(x):
        M, K = x.shape
        out = torch.zeros(M, K, dtype=torch.float64, device="cuda")
        for k in range(0, K, 32):
            b = x[:, k:k + 32].double()
            top = b.abs().max(1, keepdim=True).values
            e = torch.floor(torch.log2(torch.where(top == 0, torch.ones_like(top), top))) - 2
            unit = torch.exp2(torch.clamp(e, -127, 127))
            a, place = b.abs() / unit, torch.zeros_like(b, dtype=torch.long)
            for i in range(7):
                middle = (GRID[i] + GRID[i + 1]) / 2
                place += (a >= middle) if i % 2 else (a > middle)
            out[:, k:k + 32] = torch.copysign(grid[place], b) * unit
        return out

    code = torch.zeros(c["N"], 2 * s["wc"].shape[1], dtype=torch.long, device="cuda")
    code[:, 0::2], code[:, 1::2] = s["wc"].long() % 16, s["wc"].long() // 16
    w = grid[code % 8] * (1 - 2 * (code // 8))
    w = w * torch.exp2(s["ws"].double() - 127).repeat_interleave(32, 1)
    y = values(s["x"]) @ w[:, :c["K"]].t()
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_gradient(s):
    c = s["case"]
    kept = torch.bitwise_and(s["W"].to(torch.int32), -(1 << (8 - c["b"]))).double()
    dy = s["dy"].double()
    dx = (dy * s["sw"].double()) @ kept
    dw = (dy * s["sx"].double()[:, None]).t() @ s["codes"].double()
    return [dx, dw, torch.ones(c["M"], dtype=torch.float64, device="cuda") @ dy]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    return _exact_mx4(s) if case["op"] == "mx4" else _exact_gradient(s)
