"""Sizes of the softmax layers' operators that no kernel or no launch takes, without a GPU.  Size queries are asked before the call
is checked, so they have to answer whatever they are asked; a launch has fewer than 2^32 threads, 2^24 workgroups of 256."""
import ctypes

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


@pytest.mark.parametrize("sizes", [
    (2, 4, 2, 48, 9, 9, 4, 1), (2, 4, 2, 0, 9, 9, 4, 1), (0, 4, 2, 64, 9, 9, 4, 1), (2, 3, 2, 64, 9, 9, 4, 1), (2, 4, 2, 64, 0, 9, 4, 1),
    (2, 4, 2, 64, 9, -1, 4, 1), (2, 4, 2, 64, 9, 9, 0, 1), (2, 4, 2, 64, 9, 9, 4, -1), (1, 4, 2, 64, (1 << 30) + 1, 9, 4, 1),
    (1, 4, 2, 64, 9, (1 << 30) + 1, 4, 1), (1 << 24, 1, 1, 64, 1, 1, 4, 1), (MOST, MOST, MOST, MOST, MOST, MOST, MOST, MOST),
    # (heads x tiles with sinks: 2^64, which is 0 in 64 bits)
    (1 << 30, 1 << 30, 1 << 30, 64, 4, 1024, 4, 1024), (1 << 20, 1 << 16, 1 << 20, 64, 2, MOST, 512, MOST)])
def test_the_window_attention_query_for_sizes_that_are_refused(sizes):
    assert binding.lasad_backward_window_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("sizes", [(1, 4, 2, 48, 9000, 8000, 4), (1, 4, 3, 64, 9000, 8000, 4), (0, 4, 2, 64, 9000, 8000, 4), (1, 4, 2, 64, 9000, 0, 4),
                                   (1, 4, 2, 64, 9000, 8000, -1), (1, 4, 2, 64, 4000, 8000, 4000), (1, MOST, MOST, 64, 9000, 8000, 4)])
def test_the_step_query_for_sizes_that_are_refused(sizes):
    assert binding.lasad_decode_step_window_workspace_bytes(*sizes) == 0


by, L = ctypes.byref, binding.Layout


def _forward_qk(B, n, d=64):
    """A head each of q and k; layouts whose rows do not overlap."""
    l = L(n * d, d, d)
    return binding.load().lasad_forward_qk(0x1000, 0x2000, 0x3000, 0x4000, by(l), by(l), by(l), by(l), 1, 1, B, 1, 1, d, 1 << 15, 1 << 15, 0, n,
                                           None, None, 0, 1e-6, 2, 0, 1e4, None)


def _backward_qk(B, n, d=64):
    l = L(n * d, d, d)
    return binding.load().lasad_backward_qk(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, None, None, by(l), by(l), by(l), by(l), by(l), by(l),
                                            1, 1, B, 1, 1, d, 1 << 15, 1 << 15, 0, n, None, None, 0, 1e-6, 2, 0, 1e4, None, 0, None)


def _forward_window(B, n, m, Hq=1, Hk=1, d=64, io=1):
    q, k = L(n * Hq * d, Hq * d, d), L(m * Hk * d, Hk * d, d)
    return binding.load().lasad_forward_window(0x1000, 0x2000, 0x3000, 0x4000, None, by(q), by(k), by(k), by(q), io, io, B, Hq, Hk, d, 0, n, m, 64, 1,
                                               None, 0.125, None)


def _backward_window(B, n, m, Hq=1, Hk=1, d=64, io=1):
    q, k = L(n * Hq * d, Hq * d, d), L(m * Hk * d, Hk * d, d)
    return binding.load().lasad_backward_window(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000, by(q), by(k), by(k), by(q), by(q),
                                                by(q), by(k), by(k), io, io, B, Hq, Hk, d, 0, n, m, 64, 1, None, 0.125, 0x10000, 1 << 50, None)


def _step_window(B, Hq=1, Hk=1, d=64):
    return binding.load().lasad_decode_step_window(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 8, 1, 1, B, Hq, Hk, d, 3, None, 4, 2, 0.125, None, 0,
                                                   None)


# Every one of these has 2^24 workgroups or more (tokens of a workgroup: 8 of the norms' forward at d = 64, 32 of their backward,
# 64 or 128 queries or keys).
@pytest.mark.parametrize("call,sizes", [
    (_forward_qk, (1 << 10, 1 << 17)), (_forward_qk, (1 << 10, 1 << 16, 128)), (_forward_qk, (1 << 12, 1 << 16, 32)),
    (_backward_qk, (1 << 10, 1 << 19)), (_backward_qk, ((1 << 10) - 1, 1 << 21)),
    (_forward_window, (1 << 22, 4, 4, 4, 2)), (_forward_window, (1 << 21, 1024, 1, 1, 1)), (_forward_window, (1 << 23, 128, 1, 1, 1, 128)),
    (_forward_window, (1 << 22, 1, 1, 4, 1, 64, 0)), (_forward_window, ((1 << 24) - 3, 1, 1)),
    (_backward_window, (3 << 20, 128, 4, 4, 1)), (_backward_window, (3 << 20, 1, 512, 1, 1)), (_backward_window, (1 << 22, 1, 1, 4, 4, 64, 0)),
    (_backward_window, (9 << 20, 1, 128, 1, 1)), (_step_window, (1 << 24,)), (_step_window, (1 << 20, 16, 16)),
    # (products that pass 64 bits)
    (_forward_window, (1 << 30, 1, ((1 << 13) - 9) << 7, 1 << 15, 1 << 15)), (_backward_window, (1 << 30, 1, ((1 << 13) - 9) << 7, 1 << 15, 1 << 15)),
])
def test_more_workgroups_than_a_launch_has(call, sizes):
    assert call(*sizes) == binding.ERR_UNSUPPORTED
    assert b"launch grid" in binding.load().lasad_last_error()


def _scaled(call, scale, io):
    q, k = L(4 * 4 * 64, 4 * 64, 64), L(4 * 2 * 64, 2 * 64, 64)
    lib = binding.load()
    if call == "forward":
        return lib.lasad_forward_window(0x1000, 0x2000, 0x3000, 0x4000, None, by(q), by(k), by(k), by(q), io, io, 1, 4, 2, 64, 0, 4, 4, 64, 1, None, scale, None)
    if call == "step":
        return lib.lasad_decode_step_window(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 8, io, io, 1, 4, 2, 64, 3, None, 4, 2, scale, None, 0, None)
    return lib.lasad_backward_window(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000, by(q), by(k), by(k), by(q), by(q), by(q), by(k),
                                     by(k), io, io, 1, 4, 2, 64, 0, 4, 4, 64, 1, None, scale, 0x10000, 1 << 30, None)


@pytest.mark.parametrize("call,scale,io", [(c, 2.0 ** 127 * 1.5, io) for c in ("forward", "backward", "step") for io in (0, 1)] +
                         [("backward", s, 1) for s in (1e-37, 1e-38, 2e-39, 1e-45)])
def test_scales_that_pass_fp32_on_the_way(call, scale, io):
    """scale log2 e, and with bf16 inputs lse / scale in the backward."""
    assert _scaled(call, scale, io) == binding.ERR_UNSUPPORTED
    assert b"scale" in binding.load().lasad_last_error()
