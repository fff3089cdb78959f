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
from ._lib import Attention, Heads, check
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


def _attention(q, k, v, kv_lengths, key_mask, scale) -> Attention:
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v must be [batch, tokens, heads, dim]")
    B, SQ, H, D = q.shape
    SK, HK = k.shape[1:3]
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"q must be bfloat16 or float16, got {q.dtype}")
    _strided(q, q.dtype, q.shape, "q")
    _strided(k, q.dtype, (B, SK, HK, D), "k")
    _strided(v, q.dtype, (B, SK, HK, D), "v")
    _need(kv_lengths, torch.int32, (B,), "kv_lengths")
    if key_mask is not None:
        if key_mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("key_mask must be bool or uint8")
        _need(key_mask, key_mask.dtype, (B, SK), "key_mask")
    a = Attention()
    a.type = _TYPES[q.dtype]
    a.batch, a.heads, a.kv_heads, a.q_len, a.kv_len, a.dim = B, H, HK, SQ, SK, D
    a.scale = D ** -0.5 if scale is None else scale
    a.q, a.k, a.v = q.data_ptr(), k.data_ptr(), v.data_ptr()
    a.q_stride[:] = q.stride()[:3]
    a.k_stride[:] = k.stride()[:3]
    a.v_stride[:] = v.stride()[:3]
    a.kv_lengths, a.key_mask = _ptr(kv_lengths), _ptr(key_mask)
    return a


def attention_workspace_bytes(q: torch.Tensor, k: torch.Tensor, *, backward: bool = False) -> int:
    """Workspace with which attention (or its backward pass) of these shapes
    runs ranges of a long axis side by side."""
    a = _attention(q, k, k, None, None, None)
    return _lib.lib().tasq_attention_workspace_bytes(ctypes.byref(a), backward)


def _take_workspace(a: Attention, workspace, device, backward):
    """Sets the workspace, allocated when None and of any use; returns what
    has to live until the call has been made."""
    if workspace is None:
        nbytes = _lib.lib().tasq_attention_workspace_bytes(ctypes.byref(a), backward)
        if not nbytes:
            return None
    else:
        nbytes = workspace.numel() * workspace.element_size()
    ws = _workspace(workspace, nbytes, device, "attention")
    a.workspace, a.workspace_bytes = ws.data_ptr(), nbytes
    return ws


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *,
              kv_lengths: Optional[torch.Tensor] = None,
              key_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
              out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
              want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """(out [B, SQ, H, D], lse fp32 [B, H, SQ] or None) of softmax attention of
    queries q [B, SQ, H, D] over keys and values [B, SK, HK, D] of another
    length, bfloat16 or half at any strides that are multiples of 8; H a
    multiple of HK, whose heads are shared.  Keys count where they are below
    kv_lengths (int32 [B]) and nonzero in key_mask (bool or uint8 [B, SK]); a
    query without keys gives zeros.  scale defaults to D ** -0.5."""
    a = _attention(q, k, v, kv_lengths, key_mask, scale)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((a.batch, a.heads, a.q_len), dtype=torch.float32, device=q.device)
    _need(out, q.dtype, q.shape, "out")
    _need(lse, torch.float32, (a.batch, a.heads, a.q_len), "lse")
    a.out, a.lse = out.data_ptr(), _ptr(lse)
    ws = _take_workspace(a, workspace, q.device, 0)  # noqa: F841
    rc = _lib.lib().tasq_attention_forward(ctypes.byref(a), _stream())
    if rc:
        check(rc, "tasq_attention_forward")
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                       out: torch.Tensor, lse: torch.Tensor, *,
                       kv_lengths: Optional[torch.Tensor] = None,
                       key_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                       dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                       dv: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None):
    """Gradients (dq, dk, dv) of attention from the gradient dout of its
    output, with the out and lse that the forward call gave for the same
    arguments."""
    a = _attention(q, k, v, kv_lengths, key_mask, scale)
    _strided(dout, q.dtype, q.shape, "dout")
    _need(out, q.dtype, q.shape, "out")
    _need(lse, torch.float32, (a.batch, a.heads, a.q_len), "lse")
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    _need(dq, q.dtype, q.shape, "dq")
    _need(dk, q.dtype, k.shape, "dk")
    _need(dv, q.dtype, k.shape, "dv")
    a.out, a.lse, a.dout = out.data_ptr(), lse.data_ptr(), dout.data_ptr()
    a.dout_stride[:] = dout.stride()[:3]
    a.dq, a.dk, a.dv = dq.data_ptr(), dk.data_ptr(), dv.data_ptr()
    ws = _take_workspace(a, workspace, q.device, 1)  # noqa: F841
    rc = _lib.lib().tasq_attention_backward(ctypes.byref(a), _stream())
    if rc:
        check(rc, "tasq_attention_backward")
    return dq, dk, dv
