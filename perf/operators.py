"""Workload cases of the attention half of a quantized transformer block.

Three operators and the direction each runs in:

  linear      activations -> 8-bit codes with one scale per token, times the
              masked 8-bit weight with one scale per channel
  norm        root-mean-square norm of every head of q and k with the position
              rotation, forward or backward
  attention   softmax attention of queries over keys of another length,
              forward or backward

A case names sizes, types and layout.  ``prepare`` draws what a program has in
hand before the call (activations as slices of the projections' buffers,
weights, tables of angles, lengths of the encoder's texts); ``run`` makes one
pass; ``exact`` is the operator's definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def linear(M, K, N, b, x, y, bias=True):
    return {"op": "linear", "M": M, "K": K, "N": N, "b": b, "x": x, "y": y, "bias": bias}


def norm(B, S, H, HK, D, t, rot, pairs=False, positions=False, grad=False):
    return {"op": "norm", "B": B, "S": S, "H": H, "HK": HK, "D": D, "t": t, "rot": rot,
            "pairs": pairs, "positions": positions, "grad": grad}


def attention(B, SQ, SK, H, HK, D, t, mask="none", grad=False):
    return {"op": "attention", "B": B, "SQ": SQ, "SK": SK, "H": H, "HK": HK, "D": D, "t": t,
            "mask": mask, "grad": grad}


def listed():
    cases = {
        # the time embedding's token through a projection of the 1152-wide block
        "linear one token": linear(1, 1152, 3456, 8, "bf16", "bf16"),
        # a text of odd length into keys and values of the 640-wide UNet block
        "linear text": linear(237, 640, 1283, 6, "f16", "f16"),
        # two 1024 px images through the 1152-wide block's fused q, k, v
        "linear image": linear(8192, 1152, 3456, 5, "bf16", "bf16"),
        # the 2240-wide block with full-precision activations at both ends
        "linear wide": linear(4096, 2240, 6720, 8, "f32", "f32", bias=False),
        # one token's heads
        "norm one token": norm(1, 1, 16, 16, 72, "bf16", 72),
        # two 1024 px images' heads, image rows' positions given
        "norm image": norm(2, 4096, 16, 16, 72, "bf16", 72, positions=True),
        # its gradient for four 512 px images in the 2240-wide block
        "norm gradient": norm(4, 1024, 20, 20, 112, "f16", 112, pairs=True, grad=True),
        # one query over a long memory with shared key heads
        "attention one query": attention(2, 1, 8191, 16, 4, 128, "bf16", "lengths"),
        # image tokens over the encoder's padded texts
        "attention text": attention(2, 4096, 300, 16, 16, 72, "bf16", "lengths"),
        # image tokens among themselves, 1024 px
        "attention image": attention(2, 4096, 4096, 16, 16, 72, "bf16"),
        # gradient of image tokens over texts with some words masked
        "attention text gradient": attention(2, 4096, 300, 16, 16, 72, "bf16", "mask", grad=True),
        # gradient of image tokens among themselves, UNet block at 512 px
        "attention image gradient": attention(1, 4096, 4096, 10, 10, 64, "f16", grad=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    while True:
        kind = rng.choice(("linear", "linear", "norm", "norm gradient", "attention", "attention",
                           "one query", "attention gradient"))
        t = rng.choice(("bf16", "f16"))
        if kind == "linear":
            case = linear(_spread(rng, 1, 8192), _spread(rng, 64, 5600), _spread(rng, 32, 6720),
                          rng.randint(2, 8), rng.choice(("f32", "bf16", "f16")),
                          rng.choice(("f32", "bf16", "f16")), rng.random() < 0.5)
        elif kind.startswith("norm"):
            D = rng.choice((32, 40, 64, 72, 80, 96, 112, 128))
            HK = rng.choice((1, 2, 4, 5, 8, 16))
            case = norm(rng.randint(1, 4), _spread(rng, 1, 4096), HK * rng.choice((1, 1, 2, 4)), HK,
                        D, rng.choice(("f32", t, t)), rng.choice((0, D, D, D // 2)),
                        rng.random() < 0.5, rng.random() < 0.5, kind.endswith("gradient"))
        else:
            D = rng.choice((32, 40, 64, 72, 80, 96, 112, 128))
            HK = rng.choice((1, 2, 4, 5, 8, 16))
            G = rng.choice((1, 1, 2, 4))
            mask = rng.choice(("none", "lengths", "mask"))
            if kind == "one query":
                case = attention(rng.randint(1, 8), rng.randint(1, 4), _spread(rng, 64, 16384),
                                 HK * G, HK, D, t, mask)
            else:
                # a gradient over a handful of keys is nothing but rounding
                least = 16 if kind.endswith("gradient") else 1
                case = attention(rng.randint(1, 4), _spread(rng, 1, 4096),
                                 _spread(rng, least, 4096), HK * G, HK, D, t, mask,
                                 kind.endswith("gradient"))
        most = max(work(c)["flops"] for c in listed() if c["op"] == case["op"])
        held = max(work(c)["bytes"] for c in listed() if c["op"] == case["op"])
        if work(case)["flops"] <= most and work(case)["bytes"] <= held:
            return case


def work(case):
    c = case
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K * BYTES[c["x"]] + N * K + 8 * N + M * N * BYTES[c["y"]],
                "flops": 2 * M * N * K}
    if c["op"] == "norm":
        n = c["B"] * c["S"] * (c["H"] + c["HK"]) * c["D"]
        table = 4 * c["S"] * c["rot"]
        if c["grad"]:
            return {"bytes": 3 * n * BYTES[c["t"]] + table, "flops": 12 * n}
        return {"bytes": 2 * n * BYTES[c["t"]] + table, "flops": 7 * n}
    q, kv = c["B"] * c["SQ"] * c["H"] * c["D"], c["B"] * c["SK"] * c["HK"] * c["D"]
    products = 2 * q * c["SK"]
    if c["grad"]:
        return {"bytes": 2 * (4 * q + 4 * kv) + 4 * c["B"] * c["SQ"] * c["H"],
                "flops": 5 * products}
    return {"bytes": 2 * (2 * q + 2 * kv) + 4 * c["B"] * c["SQ"] * c["H"], "flops": 2 * products}


# ------------------------------------------------------------------- inputs

def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = case
    s = {"case": c}
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        # token magnitudes differ by a factor of ten or more, as activations' do
        spread = torch.exp(0.7 * torch.randn(M, 1, generator=g, device="cuda"))
        s["x"] = (_normal(g, M, K) * spread).to(TYPES[c["x"]])
        s["W"] = torch.clamp(torch.round(_normal(g, N, K, scale=32.0)), -128, 127).to(torch.int8)
        s["sw"] = 1e-3 + 4e-3 * torch.rand(N, generator=g, device="cuda")
        s["bias"] = _normal(g, N) if c["bias"] else None
        return s
    if c["op"] == "norm":
        B, S, H, HK, D, t = c["B"], c["S"], c["H"], c["HK"], c["D"], TYPES[c["t"]]
        # q and k are slices of the fused projection's rows
        qkv = _normal(g, B, S, (H + 2 * HK), D, dtype=t, scale=1.5)
        s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + HK]
        s["wq"], s["wk"] = (1 + 0.2 * _normal(g, D) for _ in range(2))
        s["rope"] = None
        if c["rot"]:
            half = c["rot"] // 2
            at = torch.arange(S, device="cuda", dtype=torch.float32)
            f = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float32) / half)
            ang = at[:, None] * f[None, :] + 6.28 * torch.rand(1, generator=g, device="cuda")
            pos = None
            if c["positions"]:
                pos = torch.randint(0, S, (B, S), generator=g, device="cuda", dtype=torch.int32)
            s["rope"] = (torch.cos(ang).contiguous(), torch.sin(ang).contiguous(), pos)
        if c["grad"]:
            s["dq"], s["dk"] = _normal(g, B, S, H, D, dtype=t), _normal(g, B, S, HK, D, dtype=t)
        return s
    B, SQ, SK, H, HK, D, t = (c["B"], c["SQ"], c["SK"], c["H"], c["HK"], c["D"], TYPES[c["t"]])
    s["q"] = _normal(g, B, SQ, H, D, dtype=t)
    kv = _normal(g, B, SK, 2, HK, D, dtype=t)           # the fused projection of the memory
    s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
    s["lengths"] = s["mask"] = None
    if c["mask"] == "lengths":
        s["lengths"] = torch.randint(SK // 4, SK + 1, (B,), generator=g, device="cuda",
                                     dtype=torch.int32)
    elif c["mask"] == "mask":
        s["mask"] = torch.rand(B, SK, generator=g, device="cuda") < 0.75
    if c["grad"]:
        s["do"] = _normal(g, B, SQ, H, D, dtype=t)
        s["out"], s["lse"] = _attention(s)              # kept from the forward pass
    return s


# --------------------------------------------------------------- plain forms

def _keep(s):
    """Truth values [B, 1, 1, SK] of the keys that count, or None."""
    if s["lengths"] is not None:
        at = torch.arange(s["k"].shape[1], device="cuda")
        return (at[None, :] < s["lengths"][:, None])[:, None, None, :]
    return None if s["mask"] is None else s["mask"][:, None, None, :]


def _heads(x, group=1):
    """[B, S, H, D] of any type -> fp32 [B, H * group, S, D]."""
    x = x.float().transpose(1, 2)
    return (x.repeat_interleave(group, 1) if group > 1 else x).contiguous()


def _scores(s, q, k):
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["case"]["D"] ** -0.5
    keep = _keep(s)
    return p if keep is None else p.masked_fill(~keep, -math.inf)


def _attention(s):
    c = s["case"]
    group = c["H"] // c["HK"]
    x = _scores(s, _heads(s["q"]), _heads(s["k"], group))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _heads(s["v"], group)) / torch.where(total == 0, torch.ones_like(total),
                                                               total)
    return out.transpose(1, 2).to(TYPES[c["t"]]).contiguous(), (top + torch.log(total))[..., 0]


def _attention_gradient(s):
    c = s["case"]
    group = c["H"] // c["HK"]
    q, k, v, do = _heads(s["q"]), _heads(s["k"], group), _heads(s["v"], group), _heads(s["do"])
    lse = torch.where(s["lse"] == -math.inf, torch.zeros_like(s["lse"]), s["lse"])
    p = torch.exp(_scores(s, q, k) - lse[..., None])
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * _heads(s["out"])).sum(-1, keepdim=True)) * c["D"] ** -0.5
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)

    def shared(d):
        return d.reshape(c["B"], c["HK"], group, c["SK"], c["D"]).sum(2)
    return [d.transpose(1, 2).to(TYPES[c["t"]]).contiguous() for d in (dq, shared(dk), shared(dv))]


def _angles(s):
    """cos and sin of every token, [B or 1, S, 1, R / 2]."""
    cos, sin, pos = s["rope"]
    at = torch.arange(s["q"].shape[1], device="cuda")[None] if pos is None else pos.long()
    return cos[at][:, :, None], sin[at][:, :, None]


def _rotate(s, x, back=False):
    if s["rope"] is None:
        return x
    cos, sin = _angles(s)
    sin = -sin if back else sin
    r = s["case"]["rot"]
    if s["case"]["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((y, x[..., r:]), -1)


def _norm(s, x, w):
    x32 = x.float()
    n = x32 * torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS) * w
    return _rotate(s, n).to(x.dtype).contiguous()


def _norm_gradient(s, dy, x, w):
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS)
    g = _rotate(s, dy.float(), back=True)
    n, gw = x32 * r, g * w
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx.to(x.dtype).contiguous(), (g * n).sum((0, 1, 2))


def _linear(s):
    c = s["case"]
    x = s["x"].float()
    sx = x.abs().amax(1) / 127.0
    codes = torch.round(x / torch.where(sx == 0, torch.ones_like(sx), sx)[:, None])
    step = 2 ** (8 - c["b"])
    wb = torch.floor(s["W"].float() / step) * step
    y = torch.matmul(codes.clamp(-127, 127), wb.t().contiguous()) * (sx[:, None] * s["sw"][None])
    return (y if s["bias"] is None else y + s["bias"]).to(TYPES[c["y"]])


# ----------------------------------------------------------------- one pass

def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2608_03057_amd as T
        if c["op"] == "linear":
            codes, sx = T.quantize_tokens(s["x"])
            return T.masked_linear_tokens(codes, s["W"], sx, s["sw"], c["b"], s["bias"],
                                          out_dtype=TYPES[c["y"]])
        if c["op"] == "norm":
            if c["grad"]:
                return list(T.qk_norm_rotate_backward(
                    s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], s["rope"], s["rope"],
                    eps=EPS, interleaved=c["pairs"]))
            return list(T.qk_norm_rotate(s["q"], s["k"], s["wq"], s["wk"], s["rope"], s["rope"],
                                         eps=EPS, interleaved=c["pairs"]))
        if c["grad"]:
            return list(T.attention_backward(s["do"], s["q"], s["k"], s["v"], s["out"], s["lse"],
                                             kv_lengths=s["lengths"], key_mask=s["mask"]))
        return list(T.attention(s["q"], s["k"], s["v"], kv_lengths=s["lengths"],
                                key_mask=s["mask"], want_lse=True))
    if c["op"] == "linear":
        return _linear(s)
    if c["op"] == "norm":
        if c["grad"]:
            (dq, dwq), (dk, dwk) = (_norm_gradient(s, s["dq"], s["q"], s["wq"]),
                                    _norm_gradient(s, s["dk"], s["k"], s["wk"]))
            return [dq, dk, dwq, dwk]
        return [_norm(s, s["q"], s["wq"]), _norm(s, s["k"], s["wk"])]
    return _attention_gradient(s) if c["grad"] else list(_attention(s))


# ------------------------------------------------------------ 64-bit oracle

def _exact_linear(s):
    # The codes and the token scales are fp32 decisions by definition; the sums
    # are exact.
    c, x = s["case"], s["x"].to(torch.float32)
    sx = torch.max(x.max(1).values, -x.min(1).values) / 127.0
    codes = torch.zeros_like(x)
    some = sx > 0
    codes[some] = torch.round(x[some] / sx[some, None]).clamp(-127, 127)
    kept = torch.bitwise_and(s["W"].to(torch.int32), -(1 << (8 - c["b"])))
    y = codes.double() @ kept.double().t()
    y = y * sx.double()[:, None] * s["sw"].double()
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_turn(s, x, sign):
    """Complex rotation of the first ``rot`` places by sign * angle."""
    c = s["case"]
    if s["rope"] is None:
        return x
    cos, sin, pos = s["rope"]
    z = torch.complex(cos.double(), sign * sin.double())
    z = z[:, None] if pos is None else z[pos.long()][:, :, None]
    r = c["rot"]
    i = torch.arange(0, r, 2, device="cuda") if c["pairs"] else torch.arange(r // 2, device="cuda")
    j = i + 1 if c["pairs"] else i + r // 2
    v = torch.complex(x[..., i], x[..., j]) * z
    y = x.clone()
    y[..., i], y[..., j] = v.real, v.imag
    return y


def _exact_norm(s, x, w):
    x = x.double()
    r = ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) ** -0.5
    return _exact_turn(s, x * r * w.double(), 1.0)


def _exact_norm_gradient(s, dy, x, w):
    x, w, g = x.double(), w.double(), _exact_turn(s, dy.double(), -1.0)
    D = x.shape[-1]
    m = (x ** 2).sum(-1, keepdim=True) / D + EPS
    inner = (g * w * x).sum(-1, keepdim=True)
    dx = g * w * m ** -0.5 - x * inner * m ** -1.5 / D
    return dx, (g * x * m ** -0.5).flatten(0, 2).sum(0)


def _exact_attention(s):
    """One head at a time: out, lse and, for a gradient case, dq, dk, dv."""
    c = s["case"]
    B, SQ, SK, H, HK, D = (c[n] for n in ("B", "SQ", "SK", "H", "HK", "D"))
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out, lse = torch.zeros(B, SQ, H, D, **f64), torch.full((B, H, SQ), -math.inf, **f64)
    dq, dk, dv = (torch.zeros(B, n, h, D, **f64) for n, h in ((SQ, H), (SK, HK), (SK, HK)))
    for b in range(B):
        live = torch.ones(SK, dtype=torch.bool, device="cuda")
        if s["lengths"] is not None:
            live[int(s["lengths"][b]):] = False
        if s["mask"] is not None:
            live &= s["mask"][b]
        if not bool(live.any()):
            continue
        for h in range(H):
            q = s["q"][b, :, h].double()
            k, v = (s[n][b, :, h // (H // HK)][live].double() for n in ("k", "v"))
            z = q @ k.t() / math.sqrt(D)
            lse[b, h] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            out[b, :, h] = p @ v
            if c["grad"]:
                do = s["do"][b, :, h].double()
                e = do @ v.t()
                e = p * (e - (p * e).sum(1, keepdim=True)) / math.sqrt(D)
                dq[b, :, h] = e @ k
                dk[b, live, h // (H // HK)] += e.t() @ q
                dv[b, live, h // (H // HK)] += p.t() @ do
    return [dq, dk, dv] if c["grad"] else [out, lse]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(s)
    if case["op"] == "norm":
        if case["grad"]:
            (dq, dwq), (dk, dwk) = (_exact_norm_gradient(s, s["dq"], s["q"], s["wq"]),
                                    _exact_norm_gradient(s, s["dk"], s["k"], s["wk"]))
            return [dq, dk, dwq, dwk]
        return [_exact_norm(s, s["q"], s["wq"]), _exact_norm(s, s["k"], s["wk"])]
    return _exact_attention(s)
