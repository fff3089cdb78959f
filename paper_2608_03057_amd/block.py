"""Torch-facing wrappers of the attention half of a block (argument marshalling
only): token-scaled linears, the norm and rotation of heads, attention.

As in ``api``: tensors are checked, pointers and the current stream go to the
C ABI of ``include/tasq.h``, an error raises ``TasqError``, and the work is
asynchronous on the current stream.  Outputs and workspaces are allocated
when they are not given.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import _lib
from ._lib import Heads, check
from .api import _need, _ptr, _stream

_TYPES = {torch.float32: _lib.TYPE_F32, torch.bfloat16: _lib.TYPE_BF16,
          torch.float16: _lib.TYPE_F16}

# (cos, sin, positions or None): fp32 tables [positions, rot / 2] and the
# tokens' rows of them, int32 [batch, tokens].
Rope = Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]


def _type(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return _TYPES[t.dtype]


def _strided(t: torch.Tensor, dtype, shape, name):
    """A GPU tensor with a contiguous innermost dimension and any other strides."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")


def quantize_tokens(x: torch.Tensor, out: Optional[torch.Tensor] = None,
                    scales: Optional[torch.Tensor] = None):
    """(int8 codes [M, K], fp32 scales [M]) of activations x [M, K] of any
    floating type, rows at any stride: scale max|x| * fl(1/127) per token,
    codes round(x / scale)."""
    M, K = x.shape
    _strided(x, x.dtype, x.shape, "x")
    if out is None:
        out = torch.empty((M, K), dtype=torch.int8, device=x.device)
    if scales is None:
        scales = torch.empty(M, dtype=torch.float32, device=x.device)
    _need(out, torch.int8, (M, K), "out")
    _need(scales, torch.float32, (M,), "scales")
    rc = _lib.lib().tasq_quantize_tokens(x.data_ptr(), _type(x, "x"), M, K, x.stride(0),
                                         out.data_ptr(), scales.data_ptr(), _stream())
    if rc:
        check(rc, "tasq_quantize_tokens")
    return out, scales


def masked_linear_tokens(X: torch.Tensor, W: torch.Tensor, sx: torch.Tensor, sw: torch.Tensor,
                         b: int, bias: Optional[torch.Tensor] = None, *,
                         out_dtype: torch.dtype = torch.bfloat16,
                         y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [M, N] of the masked layer on int8 codes X [M, K] with one scale per
    token (sx fp32 [M], from quantize_tokens) and per channel (sw fp32 [N]):
    (X W_b^T) sx[m] sw[n] + bias[n], W int8 [N, K] at b bits."""
    M, K = X.shape
    N = W.shape[0]
    _need(X, torch.int8, (M, K), "X")
    _need(W, torch.int8, (N, K), "W")
    _need(sx, torch.float32, (M,), "sx")
    _need(sw, torch.float32, (N,), "sw")
    _need(bias, torch.float32, (N,), "bias")
    if y is None:
        y = torch.empty((M, N), dtype=out_dtype, device=X.device)
    _need(y, y.dtype, (M, N), "y")
    rc = _lib.lib().tasq_masked_linear_tokens(X.data_ptr(), sx.data_ptr(), W.data_ptr(),
                                              sw.data_ptr(), _ptr(bias), M, N, K, int(b),
                                              y.data_ptr(), _type(y, "y"), _stream())
    if rc:
        check(rc, "tasq_masked_linear_tokens")
    return y


def _heads(j: Heads, x, weight, rope: Optional[Rope], out, name, dy=None, dweight=None):
    """Fills one tasq_heads; returns out (allocated when None)."""
    if x.dim() != 4:
        raise ValueError(f"{name} must be [batch, tokens, heads, dim]")
    _strided(x, x.dtype, x.shape, name)
    B, S, H, D = x.shape
    if out is None:
        out = torch.empty((B, S, H, D), dtype=x.dtype, device=x.device)
    _need(out, x.dtype, (B, S, H, D), f"output of {name}")
    _need(weight, torch.float32, (D,), f"weight of {name}")
    j.x, j.out, j.weight = x.data_ptr(), out.data_ptr(), _ptr(weight)
    j.x_stride[:] = x.stride()[:3]
    j.batch, j.tokens, j.heads = B, S, H
    if rope is not None:
        cos, sin, position = rope
        P, half = cos.shape
        _need(cos, torch.float32, (P, half), "cos")
        _need(sin, torch.float32, (P, half), "sin")
        _need(position, torch.int32, (B, S), "positions")
        j.cos, j.sin, j.position = cos.data_ptr(), sin.data_ptr(), _ptr(position)
        j.positions, j.rot = P, 2 * half
    if dy is not None:
        _strided(dy, x.dtype, x.shape, f"gradient of {name}")
        j.dy = dy.data_ptr()
        j.dy_stride[:] = dy.stride()[:3]
        j.dweight = _ptr(dweight)
    return out


def qk_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                   wk: Optional[torch.Tensor] = None, rope_q: Optional[Rope] = None,
                   rope_k: Optional[Rope] = None, *, eps: float = 1e-6,
                   interleaved: bool = False, out_q: Optional[torch.Tensor] = None,
                   out_k: Optional[torch.Tensor] = None):
    """(q', k') of queries q [B, S, H, D] and keys k [B, S', H', D] (or None),
    one type, any strides: root-mean-square norm of every head with weight
    [D], then the rotation of its first elements by rope = (cos, sin,
    positions).  Pairs lie rot/2 apart, or side by side with interleaved."""
    n = 1 if k is None else 2
    if k is not None and (k.dtype != q.dtype or k.shape[-1] != q.shape[-1]):
        raise ValueError("q and k differ in type or head dimension")
    jobs = (Heads * 2)()
    out_q = _heads(jobs[0], q, wq, rope_q, out_q, "q")
    if k is not None:
        out_k = _heads(jobs[1], k, wk, rope_k, out_k, "k")
    rc = _lib.lib().tasq_norm_rotate(jobs, n, _type(q, "q"), q.shape[3], eps, interleaved,
                                     _stream())
    if rc:
        check(rc, "tasq_norm_rotate")
    return out_q, out_k


def qk_norm_rotate_workspace_bytes(dim: int, n: int = 2) -> int:
    """Workspace of qk_norm_rotate_backward for n tensors of heads of dim."""
    return _lib.lib().tasq_norm_rotate_workspace_bytes(n, dim)


def _workspace(workspace, nbytes, device, name):
    if workspace is None:
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError(f"workspace of {name} must be a contiguous GPU tensor")
    return workspace


def qk_norm_rotate_backward(dq: torch.Tensor, dk: Optional[torch.Tensor], q: torch.Tensor,
                            k: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                            wk: Optional[torch.Tensor] = None, rope_q: Optional[Rope] = None,
                            rope_k: Optional[Rope] = None, *, eps: float = 1e-6,
                            interleaved: bool = False,
                            workspace: Optional[torch.Tensor] = None):
    """Gradients (dq, dk, dwq, dwk) of qk_norm_rotate from the gradients dq,
    dk of its outputs: of its inputs, in their type, and of its weights, fp32
    [D] (None where there is no weight, or no k)."""
    n = 1 if k is None else 2
    if k is not None and (k.dtype != q.dtype or k.shape[-1] != q.shape[-1]):
        raise ValueError("q and k differ in type or head dimension")
    D = q.shape[-1]
    dwq, dwk = (None if w is None else torch.empty(D, dtype=torch.float32, device=q.device)
                for w in (wq, wk))
    jobs = (Heads * 2)()
    gq = _heads(jobs[0], q, wq, rope_q, None, "q", dq, dwq)
    gk = None
    if k is not None:
        gk = _heads(jobs[1], k, wk, rope_k, None, "k", dk, dwk)
    ws = _workspace(workspace, qk_norm_rotate_workspace_bytes(D, n), q.device,
                    "qk_norm_rotate_backward")
    rc = _lib.lib().tasq_norm_rotate_backward(jobs, n, _type(q, "q"), D, eps, interleaved,
                                              ws.data_ptr(), ws.numel() * ws.element_size(),
                                              _stream())
    if rc:
        check(rc, "tasq_norm_rotate_backward")
    return gq, gk, dwq, dwk
