"""Launches of the paged cache at the border of what a launch may have: fewer than 2^32 threads along an axis."""
import pytest
import torch

from paper_2507_01652_amd import binding
from test_pages_cpu import L, _append, _step, refused

ONE = dict(Hq=1, Hk=1, lq=L(0, 64, 64), lk=L(0, 64, 64), lv=L(0, 64, 64), lo=L(0, 64, 64))


@pytest.mark.parametrize("size", [
    dict(B=1 << 23, n=1 << 23, starts=None),               # a workgroup of 512 threads a row
    dict(B=(1 << 24) - 1, n=(1 << 24) - 1, starts=None),
    dict(B=1 << 22, n=1),                                  # two a row, whatever tokens it has
    dict(B=(1 << 23) - 1, n=1)], ids=lambda s: f"{s['B']}-{s['n']}")
@pytest.mark.parametrize("queries", [True, False])
def test_append_refused(size, queries):
    refused(_append(**ONE, **size) if queries else _append(**ONE, **size, q=None, out=None))
    assert b"launch" in binding.load().lasad_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched")
def test_step_not_refused():
    """A step has a workgroup of 256 threads a row and key head."""
    assert _step(Hq=1, Hk=1, B=1 << 23) not in (binding.OK, binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)
