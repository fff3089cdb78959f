"""Torch-facing wrappers of what stands around a block's quantized linears
(argument marshalling only): the residual stream's norm with its gradient, linears
on 4-bit microscaled codes, the gradient of the token-scaled linear.

As in ``block``: tensors are checked, pointers and the current stream go to the
C ABI of ``include/tasq.h``, an error raises ``TasqError``, the work is
asynchronous on the current stream, and results carry no autograd graph.
"""
from __future__ import annotations

import functools
import struct
from typing import NamedTuple, Optional

import torch

from . import _lib
from ._lib import check
from .api import _stream
from .block import _MOST, _at, _like, _need, _strided, _too_large, _type, _workspace

_RESIDUAL = struct.Struct("7i2f4x2P4q3P3q6P4q8PN")       # tasq_residual
_KINDS = {"layer": _lib.NORM_LAYER, "rms": _lib.NORM_RMS}
_NONE = (0, 0)                  # strides of a tensor that is not there


@functools.lru_cache(maxsize=None)
def _devices() -> int:
    """Devices of the process, of which there is one where a GPU tensor is."""
    return torch.cuda.device_count()


def _here(**tensors: Optional[torch.Tensor]) -> None:
    """Calls go to the current device's stream: a tensor of another is refused.  (Of one
    device there is nothing to check: a dozen tensors take 1 us of a call's 11.)"""
    device = torch._C._cuda_getDevice()
    for name, t in tensors.items():
        if t is not None and t.get_device() != device:
            raise ValueError(f"{name} is on device {t.get_device()}, which is not the current "
                             f"device {device}")


class ResidualGrads(NamedTuple):
    """Gradients of residual_norm, None where there is no such input: of x and y
    in their type, of the rest in fp32."""
    dx: torch.Tensor
    dy: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dweight: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]
    dshift: Optional[torch.Tensor]
    dpost_weight: Optional[torch.Tensor]


def _rows(t: Optional[torch.Tensor], dtype, shape, name):
    """(address, strides of batch and token) of a [batch, tokens, width] operand."""
    if t is None:
        return 0, _NONE
    return t.data_ptr(), _strided(t, dtype, shape, name)


def _residual(x, y, gate, weight, scale, shift, post_weight, kind, residual_scale, eps):
    """(fields of a tasq_residual up to the weights, and which modulations are
    shared), checked."""
    shape, dtype = x.shape, x.dtype
    if len(shape) != 3:
        raise ValueError("x must be [batch, tokens, width]")
    B, S, C = shape
    if B > _MOST or S > _MOST or C > _MOST:
        raise _too_large(B, S, C)
    code = _type(x, "x")
    xs = _strided(x, dtype, shape, "x")
    yat, ys = _rows(y, dtype, shape, "y")
    if kind not in _KINDS:
        raise ValueError(f"kind must be 'layer' or 'rms', got {kind!r}")
    if y is None and (gate is not None or post_weight is not None or residual_scale != 1.0):
        raise ValueError("gate, post_weight and residual_scale need y")
    mod_type, shared, at, strides = None, 0, [], []
    for bit, m, name in ((1, gate, "gate"), (2, scale, "scale"), (4, shift, "shift")):
        if m is None:
            at.append(0)
            strides.append(0)
            continue
        if mod_type is None:
            mod_type = m.dtype
            if mod_type != torch.float32 and mod_type != dtype:
                raise ValueError(f"{name} must be float32 or {dtype}, got {mod_type}")
        one = m.dim() == 1
        st = _strided(m, mod_type, (C,) if one else (B, C), name)
        shared |= bit if one else 0
        at.append(m.data_ptr())
        strides.append(0 if one else st[0])
    wat = _at(weight, torch.float32, (C,), "weight")
    pat = _at(post_weight, torch.float32, (C,), "post_weight")
    if _devices() > 1:
        _here(x=x, y=y, gate=gate, weight=weight, scale=scale, shift=shift,
              post_weight=post_weight)
    return (code, _lib.TYPE_F32 if mod_type == torch.float32 else code, _KINDS[kind], shared, B, S,
            C, eps, residual_scale, x.data_ptr(), yat, xs[0], xs[1], ys[0], ys[1], *at, *strides,
            wat, pat), shared


def residual_norm(x: torch.Tensor, y: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, *,
                  weight: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  shift: Optional[torch.Tensor] = None,
                  post_weight: Optional[torch.Tensor] = None, kind: str = "layer",
                  residual_scale: float = 1.0, eps: float = 1e-6,
                  out_r: Optional[torch.Tensor] = None, out_h: Optional[torch.Tensor] = None):
    """(r, h) of a residual stream x [B, S, C] that takes a branch's output y
    through its gate and is normed for the next branch:
    r = residual_scale x + gate P(y), h = N(r) weight (1 + scale) + shift, with
    P(y) = y, or N(y) post_weight where that is given, and N the layer or the
    root-mean-square norm over C ("layer", "rms").  Without y, r is x.

    x and y of one floating type at any strides with contiguous channels; gate,
    scale and shift [B, C], or [C] for all entries, all fp32 or all of x's type;
    weight and post_weight fp32 [C]."""
    head, _ = _residual(x, y, gate, weight, scale, shift, post_weight, kind, residual_scale, eps)
    if out_h is None:
        out_h = _like(x)
    else:
        _need(out_h, x.dtype, x.shape, "out_h")
    if y is None:
        if out_r is not None:
            raise ValueError("out_r needs y: without it r is x, and is not written")
        out_r, rat = x, 0
    else:
        if out_r is None:
            out_r = _like(x)
        else:
            _need(out_r, x.dtype, x.shape, "out_r")
        rat = out_r.data_ptr()
    if _devices() > 1:
        _here(out_r=out_r, out_h=out_h)
    a = _RESIDUAL.pack(*head, rat, out_h.data_ptr(), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    rc = _lib.lib().tasq_residual_norm(a, _stream())
    if rc:
        check(rc, "tasq_residual_norm")
    return out_r, out_h


def residual_norm_workspace_bytes(x: torch.Tensor) -> int:
    """Workspace of residual_norm_backward for a stream like x [B, S, C]."""
    if max(x.shape) > _MOST:
        raise _too_large(*x.shape)
    return _lib.lib().tasq_residual_norm_workspace_bytes(_type(x, "x"), *x.shape)


def residual_norm_backward(dh: torch.Tensor, dr: Optional[torch.Tensor], r: torch.Tensor,
                           y: Optional[torch.Tensor] = None,
                           gate: Optional[torch.Tensor] = None, *,
                           weight: Optional[torch.Tensor] = None,
                           scale: Optional[torch.Tensor] = None,
                           shift: Optional[torch.Tensor] = None,
                           post_weight: Optional[torch.Tensor] = None, kind: str = "layer",
                           residual_scale: float = 1.0, eps: float = 1e-6,
                           workspace: Optional[torch.Tensor] = None) -> ResidualGrads:
    """Gradients of residual_norm from those of its outputs, dh and dr (None:
    r has no other use), with the r that the forward call gave and its other
    arguments.  Sums run in a fixed order."""
    head, shared = _residual(r, y, gate, weight, scale, shift, post_weight, kind, residual_scale,
                             eps)
    shape, dtype = r.shape, r.dtype
    hat, hs = _rows(dh, dtype, shape, "dh")
    rat, rs = _rows(dr, dtype, shape, "dr")
    if _devices() > 1:
        _here(dh=dh, dr=dr, workspace=workspace)
    dx, dy = _like(r), None if y is None else _like(r)
    B, S, C = shape
    given = (gate, scale, shift, weight, post_weight)
    grads, ats, at, nbytes = [None] * 5, [0] * 5, 0, 0
    # One buffer of all sums of a shape: an allocation takes longer than a view.
    each = [i for i in range(3) if given[i] is not None and not shared >> i & 1]
    flat = [i for i in range(5) if given[i] is not None and (i > 2 or shared >> i & 1)]
    for which, size in ((each, (len(each), B, C)), (flat, (len(flat), C))):
        if which:
            sums = torch.empty(size, dtype=torch.float32, device=r.device)
            first = sums.data_ptr()
            step = 4 * (B * C if which is each else C)
            for n, (i, view) in enumerate(zip(which, sums.unbind(0))):
                grads[i] = view
                ats[i] = first + n * step
    if each or flat:
        workspace = _workspace(
            workspace, _lib.lib().tasq_residual_norm_workspace_bytes(head[0], B, S, C), r.device,
            "residual_norm_backward")
        at, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    a = _RESIDUAL.pack(*head, 0, 0, hat, rat, hs[0], hs[1], rs[0], rs[1], dx.data_ptr(),
                       0 if dy is None else dy.data_ptr(), *ats, at, nbytes)
    rc = _lib.lib().tasq_residual_norm_backward(a, _stream())
    if rc:
        check(rc, "tasq_residual_norm_backward")
    dgate, dscale, dshift, dweight, dpost = grads
    return ResidualGrads(dx, dy, dgate, dweight, dscale, dshift, dpost)


def quantize_mx4(x: torch.Tensor, out: Optional[torch.Tensor] = None,
                 scales: Optional[torch.Tensor] = None):
    """(codes uint8 [M, K'/2], scales uint8 [M, K'/32]) of activations or a weight x
    [M, K] of any floating type, rows at any stride: 4-bit floating-point codes
    (e2m1), the even element of a pair in the low half, with one power of two for
    each 32 of a row (exponent + 127), K' = K rounded up to a multiple of 128 with
    zeros."""
    M, K = shape = x.shape
    if M > _MOST or K > _MOST:
        raise _too_large(M, K)
    st = _strided(x, x.dtype, shape, "x")
    whole = (K + 127) // 128
    if out is None:
        out = torch.empty_strided((M, 64 * whole), (64 * whole, 1), dtype=torch.uint8,
                                  device=x.device)
    else:
        _need(out, torch.uint8, (M, 64 * whole), "out")
    if scales is None:
        scales = torch.empty_strided((M, 4 * whole), (4 * whole, 1), dtype=torch.uint8,
                                     device=x.device)
    else:
        _need(scales, torch.uint8, (M, 4 * whole), "scales")
    if _devices() > 1:
        _here(x=x, out=out, scales=scales)
    rc = _lib.lib().tasq_quantize_mx4(x.data_ptr(), _type(x, "x"), M, K, st[0], out.data_ptr(),
                                      scales.data_ptr(), _stream())
    if rc:
        check(rc, "tasq_quantize_mx4")
    return out, scales


def linear_mx4(X: torch.Tensor, sx: torch.Tensor, W: torch.Tensor, sw: torch.Tensor,
               bias: Optional[torch.Tensor] = None, *, out_dtype: torch.dtype = torch.bfloat16,
               y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [M, N] = x w^T + bias of what quantize_mx4 gave for activations (X, sx) and,
    once, for a weight [N, K] (W, sw); bias fp32 [N]."""
    M, half = X.shape
    N = W.shape[0]
    if M > _MOST or N > _MOST or half > _MOST // 2:
        raise _too_large(M, N, 2 * half)
    _need(X, torch.uint8, (M, half), "X")
    _need(W, torch.uint8, (N, half), "W")
    _need(sx, torch.uint8, (M, half // 16), "sx")
    _need(sw, torch.uint8, (N, half // 16), "sw")
    if y is None:
        y = torch.empty_strided((M, N), (N, 1), dtype=out_dtype, device=X.device)
    else:
        _need(y, y.dtype, (M, N), "y")
    if _devices() > 1:
        _here(X=X, sx=sx, W=W, sw=sw, bias=bias, y=y)
    rc = _lib.lib().tasq_linear_mx4(X.data_ptr(), sx.data_ptr(), W.data_ptr(), sw.data_ptr(),
                                    _at(bias, torch.float32, (N,), "bias"), M, N, 2 * half,
                                    y.data_ptr(), _type(y, "y"), _stream())
    if rc:
        check(rc, "tasq_linear_mx4")
    return y


def masked_linear_tokens_backward_workspace_bytes(M: int, N: int, K: int) -> int:
    """Workspace with which masked_linear_tokens_backward of these sizes turns codes
    into values once where there is much work, and runs ranges of a long sum side by
    side; enough for any layout of dy.  A call with less is slower."""
    if M > _MOST or N > _MOST or K > _MOST:
        raise _too_large(M, N, K)
    return _lib.lib().tasq_masked_linear_tokens_backward_workspace_bytes(M, N, K)


def masked_linear_tokens_backward(dy: torch.Tensor, X: torch.Tensor, W: torch.Tensor,
                                  sx: torch.Tensor, sw: torch.Tensor, b: int, *,
                                  need_input: bool = True, need_weight: bool = True,
                                  dx: Optional[torch.Tensor] = None,
                                  dw: Optional[torch.Tensor] = None,
                                  dbias: Optional[torch.Tensor] = None,
                                  workspace: Optional[torch.Tensor] = None):
    """Gradients (dx [M, K], dw [N, K], dbias fp32 [N]) of masked_linear_tokens from
    that of its output, dy [M, N] bfloat16 or half with rows at any stride (below 2^22
    elements), and its arguments: the codes X with their scales sx are all that the
    program keeps of the activations.  dx is the gradient of the activations, dw that of
    the weight sw[n] W_b, both in dy's type and straight through the rounding to codes;
    the gradient of sw is (dw * W_b).sum(1).  need_input=False leaves dx out (None),
    need_weight=False dw and dbias."""
    M, N = shape = dy.shape
    K = W.shape[1]
    if M > _MOST or N > _MOST or K > _MOST:
        raise _too_large(M, N, K)
    dtype = dy.dtype
    if dtype != torch.bfloat16 and dtype != torch.float16:
        raise ValueError(f"dy must be bfloat16 or float16, got {dtype}")
    st = _strided(dy, dtype, shape, "dy")
    _need(X, torch.int8, (M, K), "X")
    _need(W, torch.int8, (N, K), "W")
    _need(sx, torch.float32, (M,), "sx")
    _need(sw, torch.float32, (N,), "sw")

    def grad(t, wanted, like, dtype, name):
        if not wanted:
            return None, 0
        if t is None:
            t = _like(like, dtype)
        else:
            _need(t, dtype, like.shape, name)
        return t, t.data_ptr()
    dx, xat = grad(dx, need_input, X, dtype, "dx")
    dw, wat = grad(dw, need_weight, W, dtype, "dw")
    dbias, bat = grad(dbias, need_weight, sw, torch.float32, "dbias")
    if _devices() > 1:
        _here(dy=dy, X=X, W=W, sx=sx, sw=sw, dx=dx, dw=dw, dbias=dbias, workspace=workspace)
    L = _lib.lib()
    if workspace is None:
        nbytes = L.tasq_masked_linear_tokens_backward_workspace_bytes(M, N, K)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    at = 0
    if nbytes:
        workspace = _workspace(workspace, nbytes, dy.device, "masked_linear_tokens_backward")
        at = workspace.data_ptr()
    rc = L.tasq_masked_linear_tokens_backward(dy.data_ptr(), _type(dy, "dy"), st[0], X.data_ptr(),
                                              sx.data_ptr(), W.data_ptr(), sw.data_ptr(), M, N, K,
                                              int(b), xat, wat, bat, at, nbytes, _stream())
    if rc:
        check(rc, "tasq_masked_linear_tokens_backward")
    return dx, dw, dbias
