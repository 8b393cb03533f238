"""Size queries of the linear-attention calls for lengths beyond every grid, without a GPU: they answer, whatever they are asked."""
import ctypes

import pytest

from paper_2507_01652_amd import binding

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("n", [(1 << 30) + 1, MOST - 62, MOST])
@pytest.mark.parametrize("B,heads,d", [(1, 1, 64), (2, 64, 64), (64, 2, 64), (1, 1, 32)])
def test_more_tokens_than_a_grid_has(B, heads, d, n):
    lib = binding.load()
    assert lib.lasad_backward_gated_workspace_bytes(B, heads, n, d) == 0
    assert lib.lasad_backward_gated_carried_workspace_bytes(B, heads, n, d) == 0
    layout = binding.Layout(0, heads * d, d)
    for io in (binding.F32, binding.BF16):
        assert lib.lasad_backward_layer_workspace_bytes(B, heads, n, d, io, ctypes.byref(layout)) == 0
        for query in (lib.lasad_forward_workspace_bytes, lib.lasad_backward_workspace_bytes, lib.lasad_backward_carried_workspace_bytes):
            query(B, heads, n, d, io)
