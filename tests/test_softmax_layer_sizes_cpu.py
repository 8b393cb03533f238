"""Size queries of the softmax layers' operators for sizes that no kernel takes, without a GPU: they are asked before the call is
checked, so they have to answer whatever they are asked."""
import pytest
import torch

from paper_2507_01652_amd import binding

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("d", [-64, 0, 1, 31, 48, 96, 256, 511, 512, 513, 1024, MOST])
def test_the_head_norms_query_for_a_head_dim_without_a_kernel(d):
    for shared in (False, True):
        assert binding.lasad_backward_qk_workspace_bytes(2, 4, 2, 16, d, shared) == 0


@pytest.mark.parametrize("sizes", [(0, 4, 2, 16), (2, 0, 2, 16), (2, 4, -1, 16), (2, 4, 2, 0), (2, 4, 2, -1), (2, 65536, 2, 16), (2, 4, MOST, 16),
                                   (1 << 16, 4, 2, 1 << 15), (MOST, MOST, MOST, MOST)])
def test_the_head_norms_query_for_other_sizes_that_are_refused(sizes):
    assert binding.lasad_backward_qk_workspace_bytes(*sizes, 64, False) == 0


@pytest.mark.parametrize("d", [48, 512, 513, 1024])
def test_the_head_norms_backward_with_a_wide_head(d):
    """Through the binding, which asks for the workspace first."""
    q, k = torch.zeros(2, 5, 4, d), torch.zeros(2, 5, 2, d)
    with pytest.raises(ValueError):
        binding.lasad_backward_qk(q, k, q, k, 3, 3)
