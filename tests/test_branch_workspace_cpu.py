"""Workspace sizes of the token-scaled linear's gradient (no GPU): room for all that
the call writes, whatever the layout of its operands."""
import pytest

import paper_2608_03057_amd as T


@pytest.mark.parametrize("M,N,K", [(520, 4456, 4408), (8192, 1152, 1152), (2048, 2240, 2400),
                                   (520, 4451, 4408), (4096, 11200, 2240)])
def test_much_work_has_room_for_values_of_all_operands(M, N, K):
    """16-bit values of W, X and dy: a dy of rows at an odd distance or address is
    copied, whether N is a multiple of 8 or not."""
    size = T.masked_linear_tokens_backward_workspace_bytes(M, N, K)
    assert size >= 2 * (N * K + M * K + M * N)


def test_little_work_has_room_for_ranges_of_both_products():
    size = T.masked_linear_tokens_backward_workspace_bytes
    assert size(8192, 128, 128) >= 2 * 128 * 128 * 4          # of tokens, for dw
    assert size(128, 8192, 128) >= 2 * 128 * 128 * 4          # of channels, for dx
    assert size(64, 64, 64) == 0                              # nothing to cut
