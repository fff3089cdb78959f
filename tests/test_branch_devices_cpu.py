"""Operands on another device than the current one are refused before anything is
enqueued, each of them by name (no GPU: tensors that only say where they are; the stream
is asked for last, and its getter stands for the call)."""
import pytest
import torch

import paper_2608_03057_amd as T
from paper_2608_03057_amd import branch


class On(torch.Tensor):
    """A CPU tensor that says it is on a GPU."""
    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


class Enqueued(Exception):
    pass


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(On)


def u8(*shape):
    return gpu(*shape, dtype=torch.uint8)


def i8(*shape):
    return gpu(*shape, dtype=torch.int8)


def bf(*shape):
    return gpu(*shape, dtype=torch.bfloat16)


def norm():
    m = {n: bf(2, 8) for n in ("gate", "scale", "shift")}
    return T.residual_norm, dict(x=bf(2, 3, 8), y=bf(2, 3, 8), weight=gpu(8), post_weight=gpu(8),
                                 out_r=bf(2, 3, 8), out_h=bf(2, 3, 8), **m)


def norm_without_branch():
    return T.residual_norm, dict(x=bf(2, 3, 8), scale=bf(8), shift=bf(8), out_h=bf(2, 3, 8))


def norm_backward():
    m = {n: bf(2, 8) for n in ("gate", "scale", "shift")}
    return T.residual_norm_backward, dict(
        dh=bf(2, 3, 8), dr=bf(2, 3, 8), r=bf(2, 3, 8), y=bf(2, 3, 8), weight=gpu(8),
        post_weight=gpu(8), workspace=u8(1 << 16), **m)


def quantize():
    return T.quantize_mx4, dict(x=bf(2, 128), out=u8(2, 64), scales=u8(2, 4))


def linear():
    return T.linear_mx4, dict(X=u8(2, 64), sx=u8(2, 4), W=u8(5, 64), sw=u8(5, 4), bias=gpu(5),
                              y=bf(2, 5))


def gradient():
    return T.masked_linear_tokens_backward, dict(
        dy=bf(4, 6), X=i8(4, 8), W=i8(6, 8), sx=gpu(4), sw=gpu(6), b=8, dx=bf(4, 8), dw=bf(6, 8),
        dbias=gpu(6), workspace=u8(256))


CALLS = (norm, norm_without_branch, norm_backward, quantize, linear, gradient)


@pytest.fixture(autouse=True)
def two_devices(monkeypatch):
    def stream():
        raise Enqueued
    monkeypatch.setattr(branch, "_stream", stream)
    monkeypatch.setattr(branch, "_devices", lambda: 2, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)


@pytest.mark.parametrize("call", CALLS)
def test_on_the_current_device(call):
    f, args = call()
    with pytest.raises(Enqueued):
        f(**args)


@pytest.mark.parametrize("call,name", [(c, n) for c in CALLS for n, t in c()[1].items()
                                       if isinstance(t, torch.Tensor)])
def test_on_another_device(call, name):
    f, args = call()
    args[name].at = 1
    # (r takes x's place in the gradient's checks.)
    shown = "x" if name == "r" else name
    with pytest.raises(ValueError, match=f"^{shown} is on .*not the current device"):
        f(**args)
