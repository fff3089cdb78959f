"""Arguments of the wrappers around a block's linears that are refused before anything
is enqueued (no GPU: tensors that only say that they are on one)."""
import pytest
import torch

import paper_2608_03057_amd as T
from paper_2608_03057_amd import branch


class On(torch.Tensor):
    is_cuda = property(lambda self: True)


def test_output_for_a_stream_without_branch_is_refused(monkeypatch):
    """r is x then, and nothing would be written to it."""
    def stream():
        raise AssertionError("enqueued")
    monkeypatch.setattr(branch, "_stream", stream)
    x, out = (torch.zeros(2, 3, 8).as_subclass(On) for _ in range(2))
    with pytest.raises(ValueError, match="out_r needs y"):
        T.residual_norm(x, out_r=out)
