"""Torch-facing wrappers of the attention half of a block (argument marshalling
only): token-scaled linears, the norm and rotation of heads, attention.

As in ``api``: tensors are checked, pointers and the current stream go to the
C ABI of ``include/tasq.h``, an error raises ``TasqError``, and the work is
asynchronous on the current stream.  Outputs and workspaces are allocated
when they are not given.  Results carry no autograd graph, whatever the inputs
require: the ``_backward`` calls give the gradients, and a program chains them.

Descriptor structs are packed with ``struct`` (0.3 us; filling a ctypes
Structure field by field takes 5): a call on one token is as long as its host
side.  The formats are those of ``_lib.Heads`` and ``_lib.Attention``.
"""
from __future__ import annotations

import struct
from typing import Optional, Tuple

import torch

from . import _lib
from ._lib import check
from .api import _need, _stream

_TYPES = {torch.float32: _lib.TYPE_F32, torch.bfloat16: _lib.TYPE_BF16,
          torch.float16: _lib.TYPE_F16}

# (cos, sin, positions or None): fp32 tables [positions, rot / 2] and the
# tokens' rows of them, int32 [batch, tokens].
Rope = Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]

_HEADS = struct.Struct("8P6q5i4x")          # tasq_heads
_ATTENTION = struct.Struct("7if3P9q5P3q4PN")    # tasq_attention


def _type(t: torch.Tensor, name: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


_MOST = 0x7fffffff          # of an int of the C ABI: ctypes would cut larger ones off


def _too_large(*sizes: int) -> ValueError:
    return ValueError(f"sizes must be below 2^31, got {sizes}")


def _strided(t: torch.Tensor, dtype, shape, name):
    """Strides of a GPU tensor with a contiguous innermost dimension."""
    st = t.stride()
    if t.is_cuda and t.dtype == dtype and t.shape == shape and st[-1] == 1:
        return st
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return st


def _at(t: Optional[torch.Tensor], dtype, shape, name) -> int:
    """Address of a contiguous GPU tensor, 0 for None."""
    if t is None:
        return 0
    _need(t, dtype, shape, name)
    return t.data_ptr()


def _like(t: torch.Tensor, dtype=None) -> torch.Tensor:
    """A contiguous tensor of t's shape, uninitialised.  (1.3 us against 2.2 of
    torch.empty with a shape, of which a call makes several.)"""
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _workspace(workspace, nbytes, device, name):
    if workspace is None:
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError(f"workspace of {name} must be a contiguous GPU tensor")
    return workspace


def quantize_tokens(x: torch.Tensor, out: Optional[torch.Tensor] = None,
                    scales: Optional[torch.Tensor] = None):
    """(int8 codes [M, K], fp32 scales [M]) of activations x [M, K] of any
    floating type, rows at any stride: scale max|x| * fl(1/127) per token,
    codes round(x / scale)."""
    M, K = shape = x.shape
    if M > _MOST or K > _MOST:
        raise _too_large(M, K)
    st = _strided(x, x.dtype, shape, "x")
    if out is None:
        out = _like(x, torch.int8)
    else:
        _need(out, torch.int8, shape, "out")
    if scales is None:
        scales = torch.empty(M, dtype=torch.float32, device=x.device)
    else:
        _need(scales, torch.float32, (M,), "scales")
    rc = _lib.lib().tasq_quantize_tokens(x.data_ptr(), _type(x, "x"), M, K, st[0],
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
    if M > _MOST or N > _MOST or K > _MOST:
        raise _too_large(M, N, K)
    _need(X, torch.int8, (M, K), "X")
    _need(W, torch.int8, (N, K), "W")
    _need(sx, torch.float32, (M,), "sx")
    _need(sw, torch.float32, (N,), "sw")
    if y is None:
        y = torch.empty_strided((M, N), (N, 1), dtype=out_dtype, device=X.device)
    else:
        _need(y, y.dtype, (M, N), "y")
    rc = _lib.lib().tasq_masked_linear_tokens(
        X.data_ptr(), sx.data_ptr(), W.data_ptr(), sw.data_ptr(),
        _at(bias, torch.float32, (N,), "bias"), M, N, K, int(b), y.data_ptr(), _type(y, "y"),
        _stream())
    if rc:
        check(rc, "tasq_masked_linear_tokens")
    return y


def _rope(rope: Optional[Rope], B: int, S: int):
    """(addresses of cos, sin and positions, rows of the tables, rotated elements)"""
    if rope is None:
        return 0, 0, 0, 0, 0
    cos, sin, position = rope
    shape = cos.shape
    positions, half = shape
    return (_at(cos, torch.float32, shape, "cos"), _at(sin, torch.float32, shape, "sin"),
            _at(position, torch.int32, (B, S), "positions"), positions, 2 * half)


def _heads(x, weight, rope: Optional[Rope], out, name, dy=None, dweight=None, like=None):
    """(a packed tasq_heads, out, what `rope` gave): out is allocated when None.
    like: (rope, its batch and tokens, what it gave) of the tensor before, which
    mostly shares them."""
    dtype, shape = x.dtype, x.shape
    if len(shape) != 4:
        raise ValueError(f"{name} must be [batch, tokens, heads, dim]")
    B, S, H, D = shape
    st = _strided(x, dtype, shape, name)
    if out is None:
        out = _like(x)
    else:
        _need(out, dtype, shape, f"output of {name}")
    if like is not None and like[0] is rope and like[1] == (B, S):
        turn = like[2]
    else:
        turn = _rope(rope, B, S)
    gat, gst, dwat = 0, (0, 0, 0, 0), 0 if dweight is None else dweight.data_ptr()
    if dy is not None:
        gst = _strided(dy, dtype, shape, f"gradient of {name}")
        gat = dy.data_ptr()
    return _HEADS.pack(x.data_ptr(), gat, out.data_ptr(),
                       _at(weight, torch.float32, (D,), f"weight of {name}"), dwat, turn[0],
                       turn[1], turn[2], st[0], st[1], st[2], gst[0], gst[1], gst[2], B, S, H,
                       turn[3], turn[4]), out, (rope, (B, S), turn)


def _same_heads(q, k):
    if k.dtype != q.dtype or k.shape[-1] != q.shape[-1]:
        raise ValueError("q and k differ in type or head dimension")


def qk_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                   wk: Optional[torch.Tensor] = None, rope_q: Optional[Rope] = None,
                   rope_k: Optional[Rope] = None, *, eps: float = 1e-6,
                   interleaved: bool = False, out_q: Optional[torch.Tensor] = None,
                   out_k: Optional[torch.Tensor] = None):
    """(q', k') of queries q [B, S, H, D] and keys k [B, S', H', D] (or None),
    one type, any strides: root-mean-square norm of every head with weight
    [D], then the rotation of its first elements by rope = (cos, sin,
    positions).  Pairs lie rot/2 apart, or side by side with interleaved."""
    jobs, out_q, turn = _heads(q, wq, rope_q, out_q, "q")
    n = 1
    if k is not None:
        _same_heads(q, k)
        more, out_k, _ = _heads(k, wk, rope_k, out_k, "k", like=turn)
        jobs, n = jobs + more, 2
    rc = _lib.lib().tasq_norm_rotate(jobs, n, _type(q, "q"), q.shape[3], eps, interleaved,
                                     _stream())
    if rc:
        check(rc, "tasq_norm_rotate")
    return out_q, out_k


def qk_norm_rotate_workspace_bytes(dim: int, n: int = 2) -> int:
    """Workspace of qk_norm_rotate_backward for n tensors of heads of dim."""
    return _lib.lib().tasq_norm_rotate_workspace_bytes(n, dim)


def qk_norm_rotate_backward(dq: torch.Tensor, dk: Optional[torch.Tensor], q: torch.Tensor,
                            k: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                            wk: Optional[torch.Tensor] = None, rope_q: Optional[Rope] = None,
                            rope_k: Optional[Rope] = None, *, eps: float = 1e-6,
                            interleaved: bool = False,
                            workspace: Optional[torch.Tensor] = None):
    """Gradients (dq, dk, dwq, dwk) of qk_norm_rotate from the gradients dq,
    dk of its outputs: of its inputs, in their type, and of its weights, fp32
    [D] (None where there is no weight, or no k)."""
    D = q.shape[-1]
    dwq, dwk = (None if w is None else torch.empty(D, dtype=torch.float32, device=q.device)
                for w in (wq, wk))
    jobs, gq, turn = _heads(q, wq, rope_q, None, "q", dq, dwq)
    n, gk = 1, None
    if k is not None:
        _same_heads(q, k)
        more, gk, _ = _heads(k, wk, rope_k, None, "k", dk, dwk, turn)
        jobs, n = jobs + more, 2
    L = _lib.lib()
    ws = _workspace(workspace, L.tasq_norm_rotate_workspace_bytes(n, D), q.device,
                    "qk_norm_rotate_backward")
    rc = L.tasq_norm_rotate_backward(jobs, n, _type(q, "q"), D, eps, interleaved, ws.data_ptr(),
                                     ws.numel() * ws.element_size(), _stream())
    if rc:
        check(rc, "tasq_norm_rotate_backward")
    return gq, gk, dwq, dwk


def _attention_head(q, k, v, kv_lengths, key_mask, scale):
    """The fields of a tasq_attention that both directions share."""
    qs, ks = q.shape, k.shape
    if len(qs) != 4 or len(ks) != 4:
        raise ValueError("q, k and v must be [batch, tokens, heads, dim]")
    B, SQ, H, D = qs
    SK, HK = ks[1], ks[2]
    dtype = q.dtype
    if dtype != torch.bfloat16 and dtype != torch.float16:
        raise ValueError(f"q must be bfloat16 or float16, got {dtype}")
    sq = _strided(q, dtype, qs, "q")
    sk = _strided(k, dtype, (B, SK, HK, D), "k")
    sv = _strided(v, dtype, ks, "v")
    mask_at = 0
    if key_mask is not None:
        if key_mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("key_mask must be bool or uint8")
        mask_at = _at(key_mask, key_mask.dtype, (B, SK), "key_mask")
    return (_TYPES[dtype], B, H, HK, SQ, SK, D, D ** -0.5 if scale is None else scale,
            q.data_ptr(), k.data_ptr(), v.data_ptr(), sq[0], sq[1], sq[2], sk[0], sk[1], sk[2],
            sv[0], sv[1], sv[2], _at(kv_lengths, torch.int32, (B,), "kv_lengths"), mask_at)


_NO_GRADS = (0, 0, 0, 0, 0, 0, 0)           # dout, its strides, dq, dk, dv


def attention_workspace_bytes(q: torch.Tensor, k: torch.Tensor, *, backward: bool = False) -> int:
    """Workspace with which attention (or its backward pass) of these shapes
    runs ranges of a long axis side by side."""
    a = _ATTENTION.pack(*_attention_head(q, k, k, None, None, None), 0, 0, *_NO_GRADS, 0, 0)
    return _lib.lib().tasq_attention_workspace_bytes(a, backward)


def _run_attention(fields, backward: bool, workspace, device, f, name):
    """Calls f with the workspace that the caller gave, or with one of the size
    that the library asks for."""
    a = _ATTENTION.pack(*fields, 0, 0)
    if workspace is None:
        nbytes = _lib.lib().tasq_attention_workspace_bytes(a, backward)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    if nbytes:
        ws = _workspace(workspace, nbytes, device, "attention")
        a = _ATTENTION.pack(*fields, ws.data_ptr(), nbytes)
    rc = f(a, _stream())
    if rc:
        check(rc, name)


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
    head = _attention_head(q, k, v, kv_lengths, key_mask, scale)
    shape = q.shape
    stats = (head[1], head[2], head[4])     # batch, heads, queries
    if out is None:
        out = _like(q)
    else:
        _need(out, q.dtype, shape, "out")
    if lse is not None:
        _need(lse, torch.float32, stats, "lse")
    elif want_lse:
        lse = torch.empty_strided(stats, (stats[1] * stats[2], stats[2], 1), dtype=torch.float32,
                                  device=q.device)
    _run_attention((*head, out.data_ptr(), 0 if lse is None else lse.data_ptr(), *_NO_GRADS),
                   False, workspace, q.device, _lib.lib().tasq_attention_forward,
                   "tasq_attention_forward")
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
    head = _attention_head(q, k, v, kv_lengths, key_mask, scale)
    shape, dtype = q.shape, q.dtype
    gs = _strided(dout, dtype, shape, "dout")
    _need(out, dtype, shape, "out")
    _need(lse, torch.float32, (head[1], head[2], head[4]), "lse")

    def grad(t, like, name):
        if t is None:
            return _like(like)
        _need(t, dtype, like.shape, name)
        return t
    dq, dk, dv = grad(dq, q, "dq"), grad(dk, k, "dk"), grad(dv, v, "dv")
    _run_attention((*head, out.data_ptr(), lse.data_ptr(), dout.data_ptr(), gs[0], gs[1], gs[2],
                    dq.data_ptr(), dk.data_ptr(), dv.data_ptr()),
                   True, workspace, q.device, _lib.lib().tasq_attention_backward,
                   "tasq_attention_backward")
    return dq, dk, dv
