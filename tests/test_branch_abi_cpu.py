"""C-ABI checks of the operators around a block's linears that need no GPU:
descriptors as the header has them, refusals before a device is touched (the
pointers below are never dereferenced on the device: each call fails its checks,
or enqueues nothing), workspace sizes."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2608_03057_amd as T
from conftest import ROOT
from paper_2608_03057_amd import _lib, branch

L = _lib.lib()
FAKE = 0x10000          # 256-byte aligned, never dereferenced
NULL, DIM, BITS = _lib.TASQ_ERR_NULL, _lib.TASQ_ERR_DIM, _lib.TASQ_ERR_BITS
OVERFLOW, RANGE, KIND = _lib.TASQ_ERR_OVERFLOW, _lib.TASQ_ERR_RANGE, _lib.TASQ_ERR_KIND
WORKSPACE, ALIGN = _lib.TASQ_ERR_WORKSPACE, _lib.TASQ_ERR_ALIGN
F32, BF16, F16 = _lib.TYPE_F32, _lib.TYPE_BF16, _lib.TYPE_F16


# ---------------------------------------------------------------- descriptors

def test_residual_layout_matches_header(tmp_path):
    py = _lib.Residual
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "tasq.h"', "int main(void){",
             'printf("size %zu\\n", sizeof(tasq_residual));']
    lines += [f'printf("{f} %zu\\n", offsetof(tasq_residual, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join([*lines, "return 0;}"]))
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src),
                           "-o", str(exe)])
    for line in filter(None, subprocess.check_output([str(exe)]).decode().split("\n")):
        field, val = line.split()
        want = ctypes.sizeof(py) if field == "size" else getattr(py, field).offset
        assert int(val) == want, (field, int(val), want)


def test_packed_residual_is_the_structure():
    """Distinct values through the packed format and back out of the structure."""
    def flat(s):
        out = []
        for f, _ in s._fields_:
            v = getattr(s, f)
            out += list(v) if isinstance(v, ctypes.Array) else [v or 0]
        return out
    values = [3 + 7 * i for i in range(len(flat(_lib.Residual())))]
    assert branch._RESIDUAL.size == ctypes.sizeof(_lib.Residual)
    assert flat(_lib.Residual.from_buffer_copy(branch._RESIDUAL.pack(*values))) == values


def test_constants_match_header():
    text = open(os.path.join(ROOT, "include", "tasq.h")).read()
    for name in ("NORM_LAYER", "NORM_RMS", "SHARED_GATE", "SHARED_SCALE", "SHARED_SHIFT"):
        assert int(re.search(rf"TASQ_{name} = (\d+)", text)[1]) == getattr(_lib, name)
    for name in ("TASQ_MAX_RESIDUAL_WIDTH", "TASQ_MAX_RESIDUAL_BATCH"):
        value = re.search(rf"#define {name} (\(?[\d <]+\)?)", text)[1]
        assert eval(value) == getattr(_lib, name)


# ------------------------------------------------------------------- refusals

def residual(**kw):
    a = _lib.Residual(type=BF16, mod_type=F32, kind=0, shared=0, batch=2, tokens=5, width=72,
                      eps=1e-6, residual_scale=1.0, x=FAKE, y=FAKE, gate=FAKE, scale=FAKE,
                      shift=FAKE, gate_stride=72, scale_stride=72, shift_stride=72, weight=FAKE,
                      post_weight=FAKE, r=FAKE, h=FAKE, dh=FAKE, dr=FAKE, dx=FAKE, dy=FAKE,
                      dgate=FAKE, dscale=FAKE, dshift=FAKE, dweight=FAKE, dpost_weight=FAKE,
                      workspace=FAKE, workspace_bytes=1 << 30)
    for s in ("x_stride", "y_stride", "dh_stride", "dr_stride"):
        getattr(a, s)[:] = (5 * 72, 72)
    for k, v in kw.items():
        if k in ("x_stride", "y_stride", "dh_stride", "dr_stride"):
            getattr(a, k)[:] = v
        else:
            setattr(a, k, v)
    return a


def forward(**kw):
    return L.tasq_residual_norm(ctypes.byref(residual(**kw)), None)


def backward(**kw):
    return L.tasq_residual_norm_backward(ctypes.byref(residual(**kw)), None)


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("kw,code", [
    (dict(type=3), KIND), (dict(type=-1), KIND), (dict(mod_type=F16), KIND),
    (dict(mod_type=5), KIND), (dict(kind=2), KIND), (dict(kind=-1), KIND),
    (dict(eps=-1.0), RANGE), (dict(eps=float("nan")), RANGE), (dict(eps=float("inf")), RANGE),
    (dict(residual_scale=float("nan")), RANGE), (dict(residual_scale=float("-inf")), RANGE),
    (dict(shared=8), RANGE), (dict(shared=-1), RANGE),
    (dict(batch=-1), DIM), (dict(tokens=-1), DIM), (dict(width=-1), DIM),
    (dict(width=_lib.TASQ_MAX_RESIDUAL_WIDTH + 1), DIM),
    (dict(batch=_lib.TASQ_MAX_RESIDUAL_BATCH + 1), DIM),
    (dict(batch=1 << 10, tokens=(1 << 20) + 1), DIM),
    (dict(x_stride=(-1, 72)), DIM), (dict(y_stride=(360, -72)), DIM),
    (dict(gate_stride=-1), DIM), (dict(scale_stride=-1), DIM), (dict(shift_stride=-1), DIM),
    (dict(x=None), NULL),
    (dict(x=FAKE + 1), ALIGN), (dict(y=FAKE + 1), ALIGN), (dict(x=FAKE + 2, type=F32), ALIGN),
    (dict(gate=FAKE + 2), ALIGN), (dict(scale=FAKE + 2), ALIGN), (dict(shift=FAKE + 1), ALIGN),
    (dict(gate=FAKE + 1, mod_type=BF16), ALIGN), (dict(weight=FAKE + 2), ALIGN),
    (dict(post_weight=FAKE + 2), ALIGN),
])
def test_residual_norm_rejects(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(r=None), NULL), (dict(h=None), NULL), (dict(h=None, y=None), NULL),
    (dict(r=FAKE + 1), ALIGN), (dict(h=FAKE + 1), ALIGN),
])
def test_residual_norm_forward_rejects(kw, code):
    assert forward(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dh=None), NULL), (dict(dx=None), NULL), (dict(dy=None), NULL),
    (dict(dh=FAKE + 1), ALIGN), (dict(dr=FAKE + 1), ALIGN), (dict(dx=FAKE + 1), ALIGN),
    (dict(dy=FAKE + 1), ALIGN), (dict(dgate=FAKE + 2), ALIGN), (dict(dscale=FAKE + 2), ALIGN),
    (dict(dshift=FAKE + 2), ALIGN), (dict(dweight=FAKE + 2), ALIGN),
    (dict(dpost_weight=FAKE + 2), ALIGN), (dict(workspace=FAKE + 16), ALIGN),
    (dict(dh_stride=(-1, 72)), DIM), (dict(dr_stride=(360, -1)), DIM),
    (dict(workspace=None), WORKSPACE),
    (dict(workspace_bytes=L.tasq_residual_norm_workspace_bytes(BF16, 2, 5, 72) - 1), WORKSPACE),
])
def test_residual_norm_backward_rejects(kw, code):
    assert backward(**kw) == code


def test_residual_norm_of_nothing():
    assert L.tasq_residual_norm(None, None) == L.tasq_residual_norm_backward(None, None) == NULL
    for kw in (dict(batch=0), dict(tokens=0), dict(width=0)):
        assert forward(x=None, y=None, r=None, h=None, **kw) == 0
        assert backward(x=None, y=None, dh=None, dr=None, dx=None, dgate=None, dscale=None,
                        dshift=None, dweight=None, dpost_weight=None, workspace=None, **kw) == 0


def test_residual_norm_workspace_bytes():
    size = L.tasq_residual_norm_workspace_bytes
    for t in (F32, BF16, F16):
        assert size(t, 2, 5, 72) >= 2 * 3 * 72 * 4 and size(t, 2, 5, 72) % (3 * 72 * 4) == 0
        # A few parts for each compute unit, however many tokens there are.
        assert size(t, 2, 1 << 20, 1152) <= 1024 * 3 * 1152 * 4
    for no in ((BF16, 0, 5, 72), (BF16, 2, 0, 72), (BF16, 2, 5, 0), (BF16, -1, 5, 72), (3, 2, 5, 72),
               (BF16, 2, 5, _lib.TASQ_MAX_RESIDUAL_WIDTH + 1)):
        assert size(*no) == 0
    x = torch.empty(2, 5, 72, dtype=torch.float16)
    assert T.residual_norm_workspace_bytes(x) == size(F16, 2, 5, 72)


def quantize_mx4(x=FAKE, t=BF16, M=4, K=32, stride=32, q=FAKE, s=FAKE):
    return L.tasq_quantize_mx4(x, t, M, K, stride, q, s, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL),
    (dict(M=-1), DIM), (dict(K=-1), DIM), (dict(stride=31), DIM), (dict(M=(1 << 30) + 1), DIM),
    (dict(K=_lib.TASQ_MAX_K + 1, stride=1 << 20), OVERFLOW),
    (dict(t=3), KIND), (dict(t=-1), KIND),
    (dict(x=FAKE + 1), ALIGN), (dict(x=FAKE + 2, t=F32), ALIGN), (dict(q=FAKE + 8), ALIGN),
    (dict(s=FAKE + 2), ALIGN),
])
def test_quantize_mx4_rejects(kw, code):
    assert quantize_mx4(**kw) == code


def linear_mx4(X=FAKE, sx=FAKE, W=FAKE, sw=FAKE, bias=None, M=4, N=4, K=128, y=FAKE, t=BF16):
    return L.tasq_linear_mx4(X, sx, W, sw, bias, M, N, K, y, t, None)


@pytest.mark.parametrize("kw,code", [
    (dict(X=None), NULL), (dict(W=None), NULL), (dict(sx=None), NULL), (dict(sw=None), NULL),
    (dict(y=None), NULL), (dict(K=0, y=None), NULL),
    (dict(M=-1), DIM), (dict(N=-1), DIM), (dict(K=-128), DIM), (dict(K=96), DIM),
    (dict(M=(1 << 30) + 1), DIM), (dict(N=(1 << 30) + 1), DIM),
    (dict(K=_lib.TASQ_MAX_K + 129), OVERFLOW), (dict(t=7), KIND),
    (dict(X=FAKE + 8), ALIGN), (dict(W=FAKE + 8), ALIGN), (dict(sx=FAKE + 2), ALIGN),
    (dict(sw=FAKE + 1), ALIGN), (dict(bias=FAKE + 2), ALIGN), (dict(y=FAKE + 1), ALIGN),
    (dict(y=FAKE + 2, t=F32), ALIGN),
])
def test_linear_mx4_rejects(kw, code):
    assert linear_mx4(**kw) == code


def test_mx4_of_nothing_is_noop():
    assert quantize_mx4(M=0, x=None, q=None, s=None) == quantize_mx4(K=0, x=None, stride=0) == 0
    assert linear_mx4(M=0, X=None, y=None) == linear_mx4(N=0, W=None, y=None) == 0


def grad(dy=FAKE, t=BF16, stride=48, X=FAKE, sx=FAKE, W=FAKE, sw=FAKE, M=4, N=48, K=32, b=8,
         dx=FAKE, dw=FAKE, dbias=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return L.tasq_masked_linear_tokens_backward(dy, t, stride, X, sx, W, sw, M, N, K, b, dx, dw,
                                                dbias, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), NULL), (dict(X=None), NULL), (dict(sx=None), NULL), (dict(W=None), NULL),
    (dict(sw=None), NULL), (dict(dw=None), NULL),
    (dict(M=-1), DIM), (dict(N=-1), DIM), (dict(K=-1), DIM), (dict(stride=47), DIM),
    (dict(M=(1 << 30) + 1), DIM), (dict(N=(1 << 30) + 1, stride=1 << 31), DIM),
    (dict(K=_lib.TASQ_MAX_K + 1), OVERFLOW), (dict(b=0), BITS), (dict(b=9), BITS),
    (dict(t=F32), KIND), (dict(t=5), KIND),
    (dict(dy=FAKE + 1), ALIGN), (dict(dx=FAKE + 1), ALIGN), (dict(dw=FAKE + 1), ALIGN),
    (dict(dbias=FAKE + 2), ALIGN), (dict(sx=FAKE + 2), ALIGN), (dict(sw=FAKE + 2), ALIGN),
    (dict(ws=FAKE + 16), ALIGN),
])
def test_token_grad_rejects(kw, code):
    assert grad(**kw) == code


def test_token_grad_rejects_rows_too_far_apart():
    text = open(os.path.join(ROOT, "include", "tasq.h")).read()
    value = re.search(r"#define TASQ_MAX_GRAD_STRIDE (\(?[\d <]+\)?)", text)[1]
    assert eval(value) == _lib.TASQ_MAX_GRAD_STRIDE
    assert grad(stride=_lib.TASQ_MAX_GRAD_STRIDE) == DIM
    assert grad(M=0, stride=_lib.TASQ_MAX_GRAD_STRIDE, dw=None, dbias=None) == 0


def test_token_grad_of_nothing_is_noop():
    assert grad(dx=None, dw=None, dbias=None) == 0
    assert grad(M=0, dw=None, dbias=None) == grad(K=0, dbias=None) == grad(M=0, N=0) == 0


def test_token_grad_workspace_bytes():
    size = T.masked_linear_tokens_backward_workspace_bytes
    assert size(8192, 128, 128) >= 2 * 128 * 128 * 4      # dw's ranges of tokens
    for no in ((-1, 8, 8), (8, -1, 8), (8, 8, -1), (8, 8, _lib.TASQ_MAX_K + 1)):
        assert size(*no) == 0


# --------------------------------------------------------------------- wrappers

def test_token_grad_wrapper_refuses():
    dy, codes, s = torch.zeros(4, 8).bfloat16(), torch.zeros(4, 8, dtype=torch.int8), torch.ones(4)
    with pytest.raises(ValueError, match="GPU tensor"):
        T.masked_linear_tokens_backward(dy, codes, codes, s, s, 8)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        T.masked_linear_tokens_backward(dy.float(), codes, codes, s, s, 8)
    big = torch.empty(1).bfloat16().expand(1, (1 << 32) + 3)
    with pytest.raises(ValueError, match="below 2\\^31"):
        T.masked_linear_tokens_backward(big, codes, codes, s, s, 8)


def test_mx4_wrappers_refuse():
    x, u = torch.zeros(4, 128), torch.zeros(4, 64, dtype=torch.uint8)
    for call in (lambda: T.quantize_mx4(x), lambda: T.linear_mx4(u, u, u, u)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    for shape in (((1 << 32) + 3, 1), (1, (1 << 32) + 3)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            T.quantize_mx4(torch.empty(1).expand(*shape))
        with pytest.raises(ValueError, match="below 2\\^31"):
            big = torch.empty(1, dtype=torch.uint8).expand(*shape)
            T.linear_mx4(big, big, big, big)


def test_residual_wrappers_refuse():
    x = torch.zeros(2, 5, 72)
    for call in (lambda: T.residual_norm(x), lambda: T.residual_norm_backward(x, x, x)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="batch, tokens, width"):
        T.residual_norm(x[0])
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        T.residual_norm(x.double())
    big = torch.empty(1).expand(1 << 31, 1, 1)
    with pytest.raises(ValueError, match="below 2\\^31"):
        T.residual_norm(big)
