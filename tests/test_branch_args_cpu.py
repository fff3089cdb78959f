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


def test_workspaces_of_sizes_past_an_int_are_refused():
    """Not answered for the size that is left of it in 32 bits."""
    far = (1 << 32) + 512
    for sizes in ((far, 512, 512), (512, far, 512), (512, 512, far)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            T.masked_linear_tokens_backward_workspace_bytes(*sizes)
    for shape in ((far, 1, 8), (1, far, 8), (1, 1, far)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            T.residual_norm_workspace_bytes(torch.empty(1).expand(*shape))
