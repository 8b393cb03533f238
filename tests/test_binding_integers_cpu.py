"""Integers beyond 32 bits in the calls of the softmax layers: refused, not cut to their low bits (no GPU, nothing is launched)."""
import pytest
import torch

from paper_2507_01652_amd import binding

B, HQ, HK, D, N = 2, 4, 2, 64, 4


class _Library:
    """In the place of liblasad: what reaches it."""
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        return lambda *a: self.called.append(name) or 0


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(binding, "_fast", lambda *a: None)                   # (as for everything that the extension does not take)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    monkeypatch.setattr(torch.Tensor, "is_pinned", lambda self: True)        # (stands for memory that a kernel can reach)
    return lib


def _call(name, **change):
    q, k = torch.zeros(B, N, HQ, D), torch.zeros(B, N, HK, D)
    q1, k1, cache = q[:, 0].contiguous(), k[:, 0].contiguous(), torch.zeros(B, HK, 9, D)
    kw = dict(forward_qk=dict(q=q, k=k, grid_h=2, grid_w=2), backward_qk=dict(q=q, k=k, d_q=q, d_k=k, grid_h=2, grid_w=2),
              decode_step_qk=dict(q=q1, k=k1, grid_h=2, grid_w=2, pos=0), forward_window=dict(q=q, k=k, v=k, window=2),
              backward_window=dict(q=q, k=k, v=k, o=q, lse=torch.zeros(B, HQ, N), d_o=q, window=2),
              decode_step_window=dict(q=q1, k=k1, v=k1, k_cache=cache, v_cache=cache.clone(), pos=0, window=2))[name]
    return getattr(binding, "lasad_" + name)(**{**kw, **change})


INTEGERS = dict(forward_qk=("grid_h", "grid_w", "start_pos", "rope", "pairing"), backward_qk=("grid_h", "grid_w", "start_pos", "rope", "pairing"),
                decode_step_qk=("grid_h", "grid_w", "pos", "rope", "pairing"), forward_window=("window", "sinks", "start_pos"),
                backward_window=("window", "sinks", "start_pos"), decode_step_window=("window", "sinks", "pos"))


@pytest.mark.parametrize("value", [1 << 31, (1 << 32) + 1, (1 << 63) - 1, -(1 << 31) - 1, (1 << 64) + 2])
@pytest.mark.parametrize("name,integer", [(n, i) for n, names in INTEGERS.items() for i in names])
def test_beyond_32_bits(library, name, integer, value):
    with pytest.raises(ValueError, match="32 bits"):
        _call(name, **{integer: value})
    assert "lasad_" + name not in library.called


@pytest.mark.parametrize("name", list(INTEGERS))
def test_what_fits_reaches_the_library(library, name):
    _call(name)
    assert library.called[-1] == "lasad_" + name
    _call(name, **{INTEGERS[name][-1]: (1 << 31) - 1})
    assert library.called[-1] == "lasad_" + name


def test_more_keys_than_32_bits_count(library):
    k = torch.zeros(B, 1, HK, D).expand(B, (1 << 32) + 3, HK, D)
    with pytest.raises(ValueError, match="32 bits"):
        _call("forward_window", k=k, v=k)
    with pytest.raises(ValueError, match="32 bits"):
        _call("backward_window", k=k, v=k, grads=(torch.zeros(B, N, HQ, D), k, k))
    q, k = (torch.zeros(B, 1, h, D).expand(B, (1 << 32) + 3, h, D) for h in (HQ, HK))
    with pytest.raises(ValueError, match="32 bits"):
        _call("forward_qk", q=q, k=k, out=(q, k))
    assert not [c for c in library.called if not c.endswith("bytes")]


@pytest.mark.parametrize("query,sizes", [("backward_qk", (2, 4, 2, 16, 64, False)), ("backward_window", (2, 4, 2, 64, 16, 16, 4, 1)),
                                         ("decode_step_window", (1, 4, 2, 64, 9000, 8000, 4))])
def test_size_queries(query, sizes):
    ask = getattr(binding, f"lasad_{query}_workspace_bytes")
    assert ask(*sizes) > 0
    for i, x in enumerate(sizes):
        if x is not False:
            with pytest.raises(ValueError, match="32 bits"):
                ask(*sizes[:i], x + (1 << 32), *sizes[i + 1:])
