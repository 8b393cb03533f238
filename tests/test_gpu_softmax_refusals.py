"""Calls of the softmax layers' operators with tensors on the GPU that no kernel takes: they raise, nothing is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [48, 512, 520, 1024])
def test_head_norms_of_a_head_dim_without_a_kernel(lasad, dtype, d):
    q, k = torch.ones(2, 6, 4, d, device="cuda", dtype=dtype), torch.ones(2, 6, 2, d, device="cuda", dtype=dtype)
    with pytest.raises(lasad.LasadError, match="head dim"):
        lasad.lasad_backward_qk(q, k, q, k, 2, 3)
    with pytest.raises(lasad.LasadError, match="head dim"):
        lasad.lasad_backward_qk(q, k, q, k, 2, 3, stream=torch.cuda.current_stream())
