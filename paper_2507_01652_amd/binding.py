"""Thin ctypes binding of liblasad's C ABI (see include/lasad.h).

Argument marshalling only: every step of the path runs in the HIP kernels.
PyTorch supplies device memory (``tensor.data_ptr()``) and the stream; there is
no CPU fallback -- a missing library is an error.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblasad.so")

F32, BF16 = 0, 1
RESET_LAST_COL, RESET_FIRST_COL, RESET_NONE = 0, 1, 2
ROPE_NONE, ROPE_1D, ROPE_2D = 0, 1, 2
PAIR_ADJACENT, PAIR_HALVES = 0, 1
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, 1, 2, 3, 4

EXPORTS = (
    "lasad_decay_factors", "lasad_forward_workspace_bytes", "lasad_forward_chunked",
    "lasad_forward_static_scratch_bytes", "lasad_forward_chunked_static",
    "lasad_decode_step", "lasad_forward_gated", "lasad_decode_step_gated",
    "lasad_forward_layer", "lasad_decode_step_layer",
    "lasad_decode_step_rows", "lasad_decode_step_cached", "lasad_decode_step_gated_cached",
    "lasad_backward_workspace_bytes", "lasad_backward_chunked",
    "lasad_backward_carried_workspace_bytes", "lasad_backward_chunked_carried",
    "lasad_backward_gated_workspace_bytes", "lasad_backward_gated",
    "lasad_backward_gated_carried_workspace_bytes", "lasad_backward_gated_carried",
    "lasad_backward_layer_workspace_bytes", "lasad_backward_layer", "lasad_backward_layer_norm",
    "lasad_forward_qk", "lasad_backward_qk_workspace_bytes", "lasad_backward_qk", "lasad_decode_step_qk",
    "lasad_forward_window", "lasad_backward_window_workspace_bytes", "lasad_backward_window",
    "lasad_decode_step_window_workspace_bytes", "lasad_decode_step_window",
    "lasad_append_pages", "lasad_forward_pages_workspace_bytes", "lasad_forward_pages",
    "lasad_decode_step_pages_workspace_bytes", "lasad_decode_step_pages",
    "lasad_last_error", "lasad_version",
)


class LasadError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"liblasad status {status}: {message}")
        self.status = status


class Layout(ctypes.Structure):
    _fields_ = [("stride_b", ctypes.c_int64), ("stride_n", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class PagesStruct(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("k_pages", "v_pages", "k_scales", "v_scales")] + [
        ("n_pages", ctypes.c_int32), ("table_pages", ctypes.c_int32), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64)]


_lib = None
_steps = None                          # the extension with the decode steps' marshalling (csrc/lasad_steps.cpp)


def load() -> ctypes.CDLL:
    """Open liblasad.so (built in-tree by ``paper_2507_01652_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2507_01652_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lp = ctypes.POINTER(Layout)
    lib.lasad_decay_factors.argtypes = [vp, ci, ci, ci, ci, ci, ci, vp, vp, vp]
    lib.lasad_decay_factors.restype = ci
    lib.lasad_forward_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.lasad_forward_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_forward_chunked.argtypes = [vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                          vp, ci, cf, vp, vp, vp, ctypes.c_size_t, vp]
    lib.lasad_forward_chunked.restype = ci
    lib.lasad_forward_static_scratch_bytes.argtypes = []
    lib.lasad_forward_static_scratch_bytes.restype = ctypes.c_size_t
    lib.lasad_forward_chunked_static.argtypes = [vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                                 vp, ci, cf, vp, vp, vp]
    lib.lasad_forward_chunked_static.restype = ci
    lib.lasad_decode_step.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp, ci, cf, vp, vp]
    lib.lasad_decode_step.restype = ci
    lib.lasad_forward_gated.argtypes = [vp, vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                        ci, cf, vp, vp, vp]
    lib.lasad_forward_gated.restype = ci
    lib.lasad_decode_step_gated.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, cf, vp, vp]
    lib.lasad_decode_step_gated.restype = ci
    lib.lasad_forward_layer.argtypes = [vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, vp, vp, vp]
    lib.lasad_forward_layer.restype = ci
    lib.lasad_decode_step_layer.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, vp, vp]
    lib.lasad_decode_step_layer.restype = ci
    lib.lasad_decode_step_rows.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, vp, ci, cf, vp, vp]
    lib.lasad_decode_step_rows.restype = ci
    lib.lasad_decode_step_cached.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, vp, ci, cf, vp]
    lib.lasad_decode_step_cached.restype = ci
    lib.lasad_decode_step_gated_cached.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci, cf, vp]
    lib.lasad_decode_step_gated_cached.restype = ci
    lib.lasad_backward_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.lasad_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_chunked.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                           vp, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_chunked.restype = ci
    lib.lasad_backward_carried_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.lasad_backward_carried_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_chunked_carried.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci,
                                                   ci, ci, vp, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_chunked_carried.restype = ci
    lib.lasad_backward_gated_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.lasad_backward_gated_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_gated.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                         ctypes.c_float, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_gated.restype = ci
    lib.lasad_backward_gated_carried_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.lasad_backward_gated_carried_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_gated_carried.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, lp, lp, ci, ci, ci, ci, ci, ci,
                                                 ci, ci, ci, ci, ctypes.c_float, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_gated_carried.restype = ci
    lib.lasad_backward_layer_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, lp]
    lib.lasad_backward_layer_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_layer.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, lp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                         ctypes.c_float, vp, ctypes.c_float, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_layer.restype = ci
    lib.lasad_backward_layer_norm.argtypes = [vp, vp, vp, vp, vp, vp, lp, lp, lp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                              ctypes.c_float, vp, ctypes.c_float, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_layer_norm.restype = ci
    lib.lasad_forward_qk.argtypes = [vp] * 4 + [lp] * 4 + [ci] * 10 + [vp, vp, ci, cf, ci, ci, cf, vp]
    lib.lasad_forward_qk.restype = ci
    lib.lasad_backward_qk_workspace_bytes.argtypes = [ci] * 6
    lib.lasad_backward_qk_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_qk.argtypes = [vp] * 8 + [lp] * 6 + [ci] * 10 + [vp, vp, ci, cf, ci, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_qk.restype = ci
    lib.lasad_decode_step_qk.argtypes = [vp] * 4 + [ci] * 9 + [vp, vp, vp, ci, cf, ci, ci, cf, vp]
    lib.lasad_decode_step_qk.restype = ci
    lib.lasad_forward_window.argtypes = [vp] * 5 + [lp] * 4 + [ci] * 11 + [vp, cf, vp]
    lib.lasad_forward_window.restype = ci
    lib.lasad_backward_window_workspace_bytes.argtypes = [ci] * 8
    lib.lasad_backward_window_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_backward_window.argtypes = [vp] * 9 + [lp] * 8 + [ci] * 11 + [vp, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_backward_window.restype = ci
    lib.lasad_decode_step_window_workspace_bytes.argtypes = [ci] * 7
    lib.lasad_decode_step_window_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_decode_step_window.argtypes = [vp] * 6 + [ci] * 8 + [vp, ci, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_decode_step_window.restype = ci
    pp = ctypes.POINTER(PagesStruct)
    lib.lasad_append_pages.argtypes = [vp] * 4 + [lp] * 4 + [pp] + [ci] * 9 + [vp, ci, vp, vp, vp, ci, cf, ci, ci, cf, vp]
    lib.lasad_append_pages.restype = ci
    lib.lasad_forward_pages_workspace_bytes.argtypes = [ci] * 9
    lib.lasad_forward_pages_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_forward_pages.argtypes = [vp] * 2 + [lp] * 2 + [pp] + [ci] * 7 + [vp, ci, vp, ci, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_forward_pages.restype = ci
    lib.lasad_decode_step_pages_workspace_bytes.argtypes = [ci] * 7
    lib.lasad_decode_step_pages_workspace_bytes.restype = ctypes.c_size_t
    lib.lasad_decode_step_pages.argtypes = [vp] * 4 + [pp] + [ci] * 9 + [vp, vp, vp, ci, cf, ci, ci, cf, ci, ci, cf, vp, ctypes.c_size_t, vp]
    lib.lasad_decode_step_pages.restype = ci
    lib.lasad_last_error.argtypes = []
    lib.lasad_last_error.restype = ctypes.c_char_p
    lib.lasad_version.argtypes = []
    lib.lasad_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != OK:
        raise LasadError(status, load().lasad_last_error().decode())


# The small calls are bound by the host: every attribute of a tensor costs 0.1 us and more, a
# stream object 2 us.  Pointers and streams therefore
# go to ctypes as plain integers, the current stream is asked for by its handle, and the checks read a tensor's
# attributes once.  The decode steps, which a program calls one after the other for every layer, do all this in an extension
# (one image through twelve layers 79 -> 48 us, 16 through 24 fused layers 147 -> 101), and so do forwards and backwards with new
# gradients on the current stream (96 sequences of 256 tokens 11.5 -> 6.7 us); what that does not take (None) goes
# through the checks here, and fails here.
_DTYPE_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _same(q: torch.Tensor, others, message: str):
    """Every tensor of `others` is contiguous and has q's shape and dtype."""
    shape, dtype = q.shape, q.dtype
    if not q.is_contiguous():
        raise ValueError(message)
    for t in others:
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(message)


def _reachable(*tensors):
    """Every tensor lies where a kernel can reach it."""
    for t in tensors:
        if t is not None and not t.is_cuda and not t.is_pinned():
            raise ValueError("tensors must be on the GPU")


def _floats(t, n: int, message: str):
    """None, or at least n fp32 values in a row."""
    if t is not None and (t.dtype != torch.float32 or not t.is_contiguous() or t.numel() < n):
        raise ValueError(message)


def extension():
    """The extension (which links to the library that load() opens); only the decode steps need it."""
    global _steps
    if _steps is None:
        load()
        try:
            from . import _steps as steps
        except ImportError as e:
            raise ImportError(f"{e}: build the extension (for the torch in use) with "
                              "`python -m paper_2507_01652_amd.build`") from e
        _steps = steps
    return _steps


def _step(name: str, *args):
    """A decode step through the extension: its output, or None where the checks here have to see the call."""
    done = getattr(_steps or extension(), name)(*args)
    if type(done) is int:
        _check(done)
    return done


def _fast(name: str, *args):
    """A forward or backward through the extension, likewise; None too where there is no extension, which these calls do
    not need."""
    if _steps is None and not _has_extension():
        return None
    done = getattr(_steps, name)(*args)
    if type(done) is int:
        _check(done)
    return done


@functools.lru_cache(maxsize=None)
def _has_extension() -> bool:
    try:
        extension()
    except ImportError:
        return False
    return True


def _handle(stream):
    return None if stream is None else stream.cuda_stream


def _scratch(nbytes: int, device, stream) -> torch.Tensor:
    """A workspace from torch's caching allocator that stays reserved until the work queued on `stream`
    (None: the current stream) has run: a block freed on another stream could be handed out again while
    the kernels still use it."""
    t = torch.empty((nbytes,), dtype=torch.uint8, device=device)
    if stream is not None and stream != torch.cuda.current_stream():
        t.record_stream(stream)
    return t


def _layout(t: torch.Tensor) -> Layout:
    """Strides of a logical [B, n, Hh, d] tensor (any permutation with unit d stride)."""
    if t.dim() == 4 and t.numel() == 0:          # no element is addressed: dense strides stand in for whatever torch reports
        return Layout(t.shape[1] * t.shape[2] * t.shape[3], t.shape[2] * t.shape[3], t.shape[3])
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("expected a [B, n_tokens, Hh, d] tensor with unit stride along d")
    return Layout(t.stride(0), t.stride(1), t.stride(2))


def version() -> str:
    return load().lasad_version().decode()


def lasad_decay_factors(gamma: torch.Tensor, grid_h: int, grid_w: int, start_pos: int, n_tokens: int,
                        boundary_mode: int = RESET_LAST_COL, want_lambda: bool = True,
                        want_cum_exp: bool = True, stream=None):
    """Decay table: returns (lambda[Hh, n] fp32 or None, cum_exp[n+1] int32 or None) on gamma's device."""
    assert gamma.dtype == torch.float32 and gamma.is_contiguous() and gamma.dim() == 1
    Hh = gamma.shape[0]
    lam = torch.empty((Hh, max(n_tokens, 0)), dtype=torch.float32, device=gamma.device) if want_lambda else None
    cum = torch.empty((max(n_tokens, 0) + 1,), dtype=torch.int32, device=gamma.device) if want_cum_exp else None
    _check(load().lasad_decay_factors(_ptr(gamma), Hh, grid_h, grid_w, start_pos, n_tokens, boundary_mode,
                                      _ptr(lam), _ptr(cum), _stream(stream)))
    return lam, cum


def lasad_forward_workspace_bytes(B: int, n_heads: int, n_tokens: int, d: int, io_dtype: int) -> int:
    return int(load().lasad_forward_workspace_bytes(B, n_heads, n_tokens, d, io_dtype))


def lasad_forward_chunked(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gamma: torch.Tensor,
                          grid_h: int, grid_w: int, start_pos: int = 0,
                          boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                          state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                          out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                          workspace: torch.Tensor | None = None, use_workspace: bool = True,
                          stream=None) -> torch.Tensor:
    """Chunked forward over positions start_pos+1 .. start_pos+n.  q, k, v: logical [B, n, Hh, d]
    views sharing one set of strides; returns o (allocated like q unless `out` is given).
    `workspace`: a device buffer of lasad_forward_workspace_bytes(...) bytes; when None one is
    taken from torch's caching allocator (use_workspace=False passes NULL: single-pass kernel)."""
    if stream is None and workspace is None and use_workspace and (out_dtype is None or out is not None):
        done = _fast("forward_chunked", q, k, v, gamma, grid_h, grid_w, start_pos, boundary_mode, q_scale, state_in, state_out, out)
        if done is not None:
            return done
    B, n, Hh, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or k.stride() != q.stride() or v.stride() != q.stride():
        raise ValueError("q, k, v must share shape and strides")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v must share a dtype")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape:
        raise ValueError("out has the wrong shape")
    for s in (state_in, state_out):
        if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or s.shape != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    assert gamma.dtype == torch.float32 and gamma.is_contiguous() and gamma.shape == (Hh,)
    lq, lo = _layout(q), _layout(out)
    if workspace is None and use_workspace and n > 0:
        need = lasad_forward_workspace_bytes(B, Hh, n, d, _dtype_code(q))
        if need:
            workspace = _scratch(need, q.device, stream)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().lasad_forward_chunked(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), ctypes.byref(lq), ctypes.byref(lo),
        _dtype_code(q), _dtype_code(out), B, Hh, d, grid_h, grid_w, start_pos, n,
        _ptr(gamma), boundary_mode, q_scale, _ptr(state_in), _ptr(state_out),
        _ptr(workspace), ws_bytes, _stream(stream)))
    return out


def lasad_forward_static_scratch_bytes() -> int:
    return int(load().lasad_forward_static_scratch_bytes())


def lasad_forward_chunked_static(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gamma: torch.Tensor,
                                 grid_h: int, grid_w: int, out: torch.Tensor, start_pos: int = 0,
                                 boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                                 state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                                 stream=None) -> torch.Tensor:
    """lasad_forward_chunked over the library's built-in scratch array: nothing is allocated, so the
    caller passes every buffer, `out` included."""
    B, n, Hh, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or k.stride() != q.stride() or v.stride() != q.stride():
        raise ValueError("q, k, v must share shape and strides")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v must share a dtype")
    if out.shape != q.shape:
        raise ValueError("out has the wrong shape")
    for s in (state_in, state_out):
        if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or s.shape != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    assert gamma.dtype == torch.float32 and gamma.is_contiguous() and gamma.shape == (Hh,)
    lq, lo = _layout(q), _layout(out)
    _check(load().lasad_forward_chunked_static(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), ctypes.byref(lq), ctypes.byref(lo),
        _dtype_code(q), _dtype_code(out), B, Hh, d, grid_h, grid_w, start_pos, n,
        _ptr(gamma), boundary_mode, q_scale, _ptr(state_in), _ptr(state_out), _stream(stream)))
    return out


def lasad_decode_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gamma: torch.Tensor,
                      state: torch.Tensor, grid_h: int, grid_w: int, pos: int,
                      boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                      out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                      stream=None) -> torch.Tensor:
    """One decode step at 0-indexed raster position `pos`.  q, k, v: contiguous [B, Hh, d];
    state: contiguous fp32 [B, Hh, d, d], updated in place.  Returns o [B, Hh, d]."""
    if out_dtype is None or out is not None:
        done = _step("decode_step", q, k, v, gamma, state, grid_h, grid_w, pos, boundary_mode, q_scale, out, _handle(stream))
        if done is not None:
            return done
    B, Hh, d = q.shape
    _same(q, (k, v), "q, k, v must be contiguous [B, Hh, d] of one dtype")
    if state.dtype != torch.float32 or not state.is_contiguous() or state.shape != (B, Hh, d, d):
        raise ValueError("state must be contiguous fp32 [B, Hh, d, d]")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    assert gamma.dtype == torch.float32 and gamma.is_contiguous() and gamma.shape == (Hh,)
    _reachable(q, k, v, gamma, state, out)
    _check(load().lasad_decode_step(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _dtype_code(q), _dtype_code(out),
                                    B, Hh, d, grid_h, grid_w, pos, _ptr(gamma), boundary_mode, q_scale,
                                    _ptr(state), _stream(stream)))
    return out


def lasad_decode_step_cached(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gamma: torch.Tensor,
                             k_cache: torch.Tensor, v_cache: torch.Tensor, grid_h: int, grid_w: int, pos: int,
                             boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                             out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                             stream=None) -> torch.Tensor:
    """The decode step at position `pos` from key / value caches (contiguous [B, Hh, T, d] of q's dtype,
    rows 0..pos-1 filled by the earlier steps; this step's k, v are appended as row pos).  Returns o."""
    B, Hh, d = q.shape
    _same(q, (k, v), "q, k, v must be contiguous [B, Hh, d] of one dtype")
    for t in (k_cache, v_cache):
        if t.dim() != 4 or tuple(t.shape[:2]) != (B, Hh) or t.shape[3] != d or t.dtype != q.dtype or not t.is_contiguous():
            raise ValueError("caches must be contiguous [B, Hh, T, d] of q's dtype")
    if k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache differ in shape")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    assert gamma.dtype == torch.float32 and gamma.is_contiguous() and gamma.shape == (Hh,)
    _check(load().lasad_decode_step_cached(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(k_cache), _ptr(v_cache),
                                           k_cache.shape[2], _dtype_code(q), _dtype_code(out), B, Hh, d,
                                           grid_h, grid_w, pos, _ptr(gamma), boundary_mode, q_scale, _stream(stream)))
    return out


def lasad_decode_step_gated_cached(q: torch.Tensor, lam: torch.Tensor, v: torch.Tensor,
                                   lam_cache: torch.Tensor, v_cache: torch.Tensor, grid_h: int, grid_w: int, pos: int,
                                   k: torch.Tensor | None = None, k_cache: torch.Tensor | None = None,
                                   boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                                   out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                                   stream=None) -> torch.Tensor:
    """The vector-decay decode step at position `pos` from caches of the gate rows and of v (and of k with an own
    key; contiguous [B, Hh, T, d] of q's dtype, rows 0..pos-1 filled by the earlier steps; this step's rows are
    appended as row pos).  Returns o."""
    B, Hh, d = q.shape
    if (k is None) != (k_cache is None):
        raise ValueError("k and k_cache go together")
    _same(q, (lam, v) if k is None else (lam, v, k), "q, lam, k, v must be contiguous [B, Hh, d] of one dtype")
    for t in (lam_cache, v_cache) + (() if k_cache is None else (k_cache,)):
        if t.dim() != 4 or tuple(t.shape[:2]) != (B, Hh) or t.shape[3] != d or t.dtype != q.dtype or not t.is_contiguous():
            raise ValueError("caches must be contiguous [B, Hh, T, d] of q's dtype")
        if t.shape != lam_cache.shape:
            raise ValueError("the caches differ in shape")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    _check(load().lasad_decode_step_gated_cached(_ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(out),
                                                 _ptr(lam_cache), _ptr(k_cache), _ptr(v_cache), lam_cache.shape[2],
                                                 _dtype_code(q), _dtype_code(out), B, Hh, d,
                                                 grid_h, grid_w, pos, boundary_mode, q_scale, _stream(stream)))
    return out


def lasad_forward_gated(q: torch.Tensor, lam: torch.Tensor, v: torch.Tensor, grid_h: int, grid_w: int,
                        k: torch.Tensor | None = None, start_pos: int = 0,
                        boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                        state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                        stream=None) -> torch.Tensor:
    """Vector-decay forward (Section 3.4 as written).  q, lam, v (and k, or None for k = 1 - lam):
    logical [B, n, Hh, d] views sharing one set of strides; returns o."""
    if stream is None and (out_dtype is None or out is not None):
        done = _fast("forward_gated", q, lam, v, grid_h, grid_w, k, start_pos, boundary_mode, q_scale, state_in, state_out, out)
        if done is not None:
            return done
    B, n, Hh, d = q.shape
    for t in (lam, v) + (() if k is None else (k,)):
        if t.shape != q.shape or t.stride() != q.stride() or t.dtype != q.dtype:
            raise ValueError("q, lam, k, v must share shape, strides and dtype")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape:
        raise ValueError("out has the wrong shape")
    for s in (state_in, state_out):
        if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or s.shape != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    lq, lo = _layout(q), _layout(out)
    _check(load().lasad_forward_gated(
        _ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(out), ctypes.byref(lq), ctypes.byref(lo),
        _dtype_code(q), _dtype_code(out), B, Hh, d, grid_h, grid_w, start_pos, n,
        boundary_mode, q_scale, _ptr(state_in), _ptr(state_out), _stream(stream)))
    return out


def lasad_decode_step_gated(q: torch.Tensor, lam: torch.Tensor, v: torch.Tensor, state: torch.Tensor,
                            grid_h: int, grid_w: int, pos: int, k: torch.Tensor | None = None,
                            boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                            out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                            stream=None) -> torch.Tensor:
    """One vector-decay decode step.  q, lam, v (k): contiguous [B, Hh, d]; state fp32 [B, Hh, d, d] in place."""
    if out_dtype is None or out is not None:
        done = _step("decode_step_gated", q, lam, v, state, grid_h, grid_w, pos, k, boundary_mode, q_scale, out, _handle(stream))
        if done is not None:
            return done
    B, Hh, d = q.shape
    _same(q, (lam, v) if k is None else (lam, v, k), "q, lam, k, v must be contiguous [B, Hh, d] of one dtype")
    if state.dtype != torch.float32 or not state.is_contiguous() or state.shape != (B, Hh, d, d):
        raise ValueError("state must be contiguous fp32 [B, Hh, d, d]")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    _reachable(q, lam, k, v, state, out)
    _check(load().lasad_decode_step_gated(_ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(out),
                                          _dtype_code(q), _dtype_code(out), B, Hh, d, grid_h, grid_w, pos,
                                          boundary_mode, q_scale, _ptr(state), _stream(stream)))
    return out


def lasad_forward_layer(q_pre: torch.Tensor, z: torch.Tensor, v: torch.Tensor, grid_h: int, grid_w: int,
                        norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                        start_pos: int = 0, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                        state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                        stream=None) -> torch.Tensor:
    """Algorithm 1 between its Linear maps: SiLU(q_pre), sigmoid(z), k = 1 - lambda, recurrence, RMS norm.
    q_pre, z, v: logical [B, n, Hh, 64] views sharing strides; norm_eps < 0 switches the norm off."""
    if stream is None and (out_dtype is None or out is not None):
        done = _fast("forward_layer", q_pre, z, v, grid_h, grid_w, norm_weight, norm_eps, start_pos, boundary_mode, q_scale, state_in,
                     state_out, out)
        if done is not None:
            return done
    B, n, Hh, d = q_pre.shape
    for t in (z, v):
        if t.shape != q_pre.shape or t.stride() != q_pre.stride() or t.dtype != q_pre.dtype:
            raise ValueError("q_pre, z, v must share shape, strides and dtype")
    if norm_weight is not None and (norm_weight.dtype != torch.float32 or not norm_weight.is_contiguous()
                                    or norm_weight.numel() != Hh * d):
        raise ValueError("norm_weight must be contiguous fp32 [Hh, d]")
    if out is None:
        out = torch.empty_like(q_pre, dtype=out_dtype or q_pre.dtype)
    for s in (state_in, state_out):
        if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or s.shape != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    lq, lo = _layout(q_pre), _layout(out)
    _check(load().lasad_forward_layer(
        _ptr(q_pre), _ptr(z), _ptr(v), _ptr(out), ctypes.byref(lq), ctypes.byref(lo),
        _dtype_code(q_pre), _dtype_code(out), B, Hh, d, grid_h, grid_w, start_pos, n,
        boundary_mode, q_scale, _ptr(norm_weight), norm_eps, _ptr(state_in), _ptr(state_out), _stream(stream)))
    return out


def lasad_decode_step_layer(q_pre: torch.Tensor, z: torch.Tensor, v: torch.Tensor, state: torch.Tensor,
                            grid_h: int, grid_w: int, pos: int, norm_weight: torch.Tensor | None = None,
                            norm_eps: float = 1e-6, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                            out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                            stream=None) -> torch.Tensor:
    """One decode step of the fused layer.  q_pre, z, v: contiguous [B, Hh, d]; state fp32 in place."""
    if out_dtype is None or out is not None:
        done = _step("decode_step_layer", q_pre, z, v, state, grid_h, grid_w, pos, norm_weight, norm_eps, boundary_mode, q_scale, out,
                     _handle(stream))
        if done is not None:
            return done
    B, Hh, d = q_pre.shape
    _same(q_pre, (z, v), "q_pre, z, v must be contiguous [B, Hh, d] of one dtype")
    if state.dtype != torch.float32 or not state.is_contiguous() or state.shape != (B, Hh, d, d):
        raise ValueError("state must be contiguous fp32 [B, Hh, d, d]")
    if out is None:
        out = torch.empty_like(q_pre, dtype=out_dtype or q_pre.dtype)
    elif out.numel() < q_pre.numel() or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    _floats(norm_weight, Hh * d, "norm_weight must be contiguous fp32 [Hh, d]")
    _reachable(q_pre, z, v, state, norm_weight, out)
    _check(load().lasad_decode_step_layer(_ptr(q_pre), _ptr(z), _ptr(v), _ptr(out), _dtype_code(q_pre), _dtype_code(out),
                                          B, Hh, d, grid_h, grid_w, pos, boundary_mode, q_scale,
                                          _ptr(norm_weight), norm_eps, _ptr(state), _stream(stream)))
    return out


def lasad_decode_step_rows(q: torch.Tensor, v: torch.Tensor, state: torch.Tensor, pos_rows: torch.Tensor,
                           grid_h: int, grid_w: int, k: torch.Tensor | None = None,
                           lam: torch.Tensor | None = None, gamma: torch.Tensor | None = None,
                           boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                           out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                           stream=None) -> torch.Tensor:
    """One decode step with a raster position per batch row (pos_rows: int32 [B] on the device; entries
    outside the grid mark inactive rows).  Scalar decay: give gamma and k; vector decay: give lam (k optional)."""
    if out_dtype is None or out is not None:
        done = _step("decode_step_rows", q, v, state, pos_rows, grid_h, grid_w, k, lam, gamma, boundary_mode, q_scale, out,
                     _handle(stream))
        if done is not None:
            return done
    B, Hh, d = q.shape
    _same(q, [x for x in (v, k, lam) if x is not None], "q, lam, k, v must be contiguous [B, Hh, d] of one dtype")
    if state.dtype != torch.float32 or not state.is_contiguous() or state.shape != (B, Hh, d, d):
        raise ValueError("state must be contiguous fp32 [B, Hh, d, d]")
    if pos_rows.dtype != torch.int32 or pos_rows.numel() != B or not pos_rows.is_contiguous():
        raise ValueError("pos_rows must be contiguous int32 [B]")
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hh, d]")
    _floats(gamma, Hh, "gamma must be contiguous fp32 [Hh]")
    _reachable(q, lam, k, v, state, pos_rows, gamma, out)
    _check(load().lasad_decode_step_rows(_ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(out),
                                         _dtype_code(q), _dtype_code(out), B, Hh, d, grid_h, grid_w,
                                         _ptr(pos_rows), _ptr(gamma), boundary_mode, q_scale, _ptr(state),
                                         _stream(stream)))
    return out


def lasad_backward_workspace_bytes(B: int, n_heads: int, n_tokens: int, d: int, io_dtype: int) -> int:
    return int(load().lasad_backward_workspace_bytes(B, n_heads, n_tokens, d, io_dtype))


def lasad_backward_chunked(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, d_o: torch.Tensor,
                           gamma: torch.Tensor, grid_h: int, grid_w: int, start_pos: int = 0,
                           boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                           grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                           dgamma: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                           stream=None):
    """Gradients of lasad_forward_chunked (zero initial state).  q, k, v, d_o: logical [B, n, Hh, d]
    views sharing strides and dtype.  Returns (dq, dk, dv, dgamma); `grads` may give the three
    output tensors (sharing one set of strides), `workspace` a uint8 device tensor."""
    if grads is None and grad_dtype is None and dgamma is None and workspace is None and stream is None:
        done = _fast("backward_chunked", q, k, v, d_o, gamma, grid_h, grid_w, start_pos, boundary_mode, q_scale)
        if done is not None:
            return done
    B, n, Hh, d = q.shape
    for t in (k, v, d_o):
        if t.shape != q.shape or t.stride() != q.stride() or t.dtype != q.dtype:
            raise ValueError("q, k, v, d_o must share shape, strides and dtype")
    if grads is None:
        grads = tuple(torch.empty_like(q, dtype=grad_dtype or q.dtype) for _ in range(3))
    dq, dk, dv = grads
    for t in (dk, dv):
        if t.shape != q.shape or t.stride() != dq.stride() or t.dtype != dq.dtype:
            raise ValueError("dq, dk, dv must share shape, strides and dtype")
    if dq.shape != q.shape:
        raise ValueError("gradient tensors have the wrong shape")
    if gamma.dtype != torch.float32 or gamma.numel() != Hh or not gamma.is_contiguous():
        raise ValueError("gamma must be contiguous fp32 [Hh]")
    if dgamma is None:
        dgamma = torch.empty((Hh,), dtype=torch.float32, device=q.device)
    need = lasad_backward_workspace_bytes(B, Hh, n, d, _dtype_code(q))
    if workspace is None and need:
        workspace = _scratch(need, q.device, stream)
    li, lg = _layout(q), _layout(dq)
    _check(load().lasad_backward_chunked(
        _ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgamma),
        ctypes.byref(li), ctypes.byref(lg), _dtype_code(q), _dtype_code(dq),
        B, Hh, d, grid_h, grid_w, start_pos, n, _ptr(gamma), boundary_mode, q_scale,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return dq, dk, dv, dgamma


def lasad_backward_carried_workspace_bytes(B: int, n_heads: int, n_tokens: int, d: int, io_dtype: int) -> int:
    return int(load().lasad_backward_carried_workspace_bytes(B, n_heads, n_tokens, d, io_dtype))


def lasad_backward_chunked_carried(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, d_o: torch.Tensor,
                                   gamma: torch.Tensor, grid_h: int, grid_w: int,
                                   state_in: torch.Tensor | None = None, d_state_out: torch.Tensor | None = None,
                                   start_pos: int = 0, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                                   grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                                   dgamma: torch.Tensor | None = None, d_state_in: torch.Tensor | None = None,
                                   workspace: torch.Tensor | None = None, stream=None):
    """lasad_backward_chunked for a call that starts from state_in and whose final state enters the loss with
    gradient d_state_out (fp32 [B, Hh, d, d] each, or None).  Returns (dq, dk, dv, dgamma, d_state_in)."""
    B, n, Hh, d = q.shape
    for t in (k, v, d_o):
        if t.shape != q.shape or t.stride() != q.stride() or t.dtype != q.dtype:
            raise ValueError("q, k, v, d_o must share shape, strides and dtype")
    if grads is None:
        grads = tuple(torch.empty_like(q, dtype=grad_dtype or q.dtype) for _ in range(3))
    dq, dk, dv = grads
    for t in (dk, dv):
        if t.shape != q.shape or t.stride() != dq.stride() or t.dtype != dq.dtype:
            raise ValueError("dq, dk, dv must share shape, strides and dtype")
    for st in (state_in, d_state_out, d_state_in):
        if st is not None and (st.dtype != torch.float32 or not st.is_contiguous() or tuple(st.shape) != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    if gamma.dtype != torch.float32 or gamma.numel() != Hh or not gamma.is_contiguous():
        raise ValueError("gamma must be contiguous fp32 [Hh]")
    if dgamma is None:
        dgamma = torch.empty((Hh,), dtype=torch.float32, device=q.device)
    if d_state_in is None:
        d_state_in = torch.empty((B, Hh, d, d), dtype=torch.float32, device=q.device)
    need = lasad_backward_carried_workspace_bytes(B, Hh, n, d, _dtype_code(q))
    if workspace is None and need:
        workspace = _scratch(need, q.device, stream)
    li, lg = _layout(q), _layout(dq)
    _check(load().lasad_backward_chunked_carried(
        _ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(state_in), _ptr(d_state_out),
        _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgamma), _ptr(d_state_in),
        ctypes.byref(li), ctypes.byref(lg), _dtype_code(q), _dtype_code(dq),
        B, Hh, d, grid_h, grid_w, start_pos, n, _ptr(gamma), boundary_mode, q_scale,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return dq, dk, dv, dgamma, d_state_in


def lasad_backward_gated_workspace_bytes(B: int, n_heads: int, n_tokens: int, d: int) -> int:
    return int(load().lasad_backward_gated_workspace_bytes(B, n_heads, n_tokens, d))


def lasad_backward_gated(q: torch.Tensor, lam: torch.Tensor, v: torch.Tensor, d_o: torch.Tensor,
                         grid_h: int, grid_w: int, k: torch.Tensor | None = None, start_pos: int = 0,
                         boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                         grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                         workspace: torch.Tensor | None = None, stream=None):
    """Gradients of lasad_forward_gated (zero initial state).  q, lam, v, d_o (and k, or None for the
    tied key): logical [B, n, Hh, d] views sharing strides and dtype.  Returns (dq, dlam, dv) with the
    tied key, (dq, dlam, dv, dk) with an own key; `grads` may give these output tensors (sharing one set
    of strides), `workspace` a uint8 device tensor."""
    if grads is None and grad_dtype is None and workspace is None and stream is None:
        done = _fast("backward_gated", q, lam, v, d_o, grid_h, grid_w, k, start_pos, boundary_mode, q_scale)
        if done is not None:
            return done
    B, n, Hh, d = q.shape
    for t in (lam, v, d_o) + (() if k is None else (k,)):
        if t.shape != q.shape or t.stride() != q.stride() or t.dtype != q.dtype:
            raise ValueError("q, lam, k, v, d_o must share shape, strides and dtype")
    if grads is None:
        grads = tuple(torch.empty_like(q, dtype=grad_dtype or q.dtype) for _ in range(3 if k is None else 4))
    if len(grads) != (3 if k is None else 4):
        raise ValueError("grads must hold dq, dlam, dv (and dk with an own key)")
    dq, dlam, dv = grads[:3]
    dk = None if k is None else grads[3]
    for t in grads:
        if t.shape != q.shape or t.stride() != dq.stride() or t.dtype != dq.dtype:
            raise ValueError("gradient tensors must share q's shape and one set of strides and dtype")
    need = lasad_backward_gated_workspace_bytes(B, Hh, n, d)
    if workspace is None and need:
        workspace = _scratch(need, q.device, stream)
    li, lg = _layout(q), _layout(dq)
    _check(load().lasad_backward_gated(
        _ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(d_o), _ptr(dq), _ptr(dlam), _ptr(dk), _ptr(dv),
        ctypes.byref(li), ctypes.byref(lg), _dtype_code(q), _dtype_code(dq),
        B, Hh, d, grid_h, grid_w, start_pos, n, boundary_mode, q_scale,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return (dq, dlam, dv) if k is None else (dq, dlam, dv, dk)


def lasad_backward_gated_carried_workspace_bytes(B: int, n_heads: int, n_tokens: int, d: int) -> int:
    return int(load().lasad_backward_gated_carried_workspace_bytes(B, n_heads, n_tokens, d))


def lasad_backward_gated_carried(q: torch.Tensor, lam: torch.Tensor, v: torch.Tensor, d_o: torch.Tensor,
                                 grid_h: int, grid_w: int, k: torch.Tensor | None = None,
                                 state_in: torch.Tensor | None = None, d_state_out: torch.Tensor | None = None,
                                 start_pos: int = 0, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                                 grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                                 d_state_in: torch.Tensor | None = None,
                                 workspace: torch.Tensor | None = None, stream=None):
    """lasad_backward_gated for a call that starts from state_in and whose final state enters the loss with gradient
    d_state_out (fp32 [B, Hh, d, d] each, or None).  Returns (dq, dlam, dv[, dk], d_state_in)."""
    B, n, Hh, d = q.shape
    for t in (lam, v, d_o) + (() if k is None else (k,)):
        if t.shape != q.shape or t.stride() != q.stride() or t.dtype != q.dtype:
            raise ValueError("q, lam, k, v, d_o must share shape, strides and dtype")
    if grads is None:
        grads = tuple(torch.empty_like(q, dtype=grad_dtype or q.dtype) for _ in range(3 if k is None else 4))
    if len(grads) != (3 if k is None else 4):
        raise ValueError("grads must hold dq, dlam, dv (and dk with an own key)")
    dq, dlam, dv = grads[:3]
    dk = None if k is None else grads[3]
    for t in grads:
        if t.shape != q.shape or t.stride() != dq.stride() or t.dtype != dq.dtype:
            raise ValueError("gradient tensors must share q's shape and one set of strides and dtype")
    for st in (state_in, d_state_out, d_state_in):
        if st is not None and (st.dtype != torch.float32 or not st.is_contiguous() or tuple(st.shape) != (B, Hh, d, d)):
            raise ValueError("states must be contiguous fp32 [B, Hh, d, d]")
    if d_state_in is None:
        d_state_in = torch.empty((B, Hh, d, d), dtype=torch.float32, device=q.device)
    need = lasad_backward_gated_carried_workspace_bytes(B, Hh, n, d)
    if workspace is None and need:
        workspace = _scratch(need, q.device, stream)
    li, lg = _layout(q), _layout(dq)
    _check(load().lasad_backward_gated_carried(
        _ptr(q), _ptr(lam), _ptr(k), _ptr(v), _ptr(d_o), _ptr(state_in), _ptr(d_state_out),
        _ptr(dq), _ptr(dlam), _ptr(dk), _ptr(dv), _ptr(d_state_in),
        ctypes.byref(li), ctypes.byref(lg), _dtype_code(q), _dtype_code(dq),
        B, Hh, d, grid_h, grid_w, start_pos, n, boundary_mode, q_scale,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return ((dq, dlam, dv) if k is None else (dq, dlam, dv, dk)) + (d_state_in,)


def lasad_backward_layer_workspace_bytes(q_pre: torch.Tensor) -> int:
    B, n, Hh, d = q_pre.shape
    lq = _layout(q_pre)
    return int(load().lasad_backward_layer_workspace_bytes(B, Hh, n, d, _dtype_code(q_pre), ctypes.byref(lq)))


def lasad_backward_layer(q_pre: torch.Tensor, z: torch.Tensor, v: torch.Tensor, d_out: torch.Tensor,
                         grid_h: int, grid_w: int, norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                         start_pos: int = 0, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                         grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                         dweight: torch.Tensor | None = None, want_dweight: bool = True,
                         workspace: torch.Tensor | None = None, stream=None):
    """Gradients of lasad_forward_layer (zero initial state).  q_pre, z, v: logical [B, n, Hh, 64] views
    sharing strides and dtype; d_out of the same shape and dtype with strides of its own.  Returns
    (dq_pre, dz, dv, dweight); dweight is fp32 [Hh, d], or None with want_dweight=False."""
    if grads is None and grad_dtype is None and dweight is None and workspace is None and stream is None:
        done = _fast("backward_layer", q_pre, z, v, d_out, grid_h, grid_w, norm_weight, norm_eps, start_pos, boundary_mode, q_scale,
                     want_dweight)
        if done is not None:
            return done
    B, n, Hh, d = q_pre.shape
    for t in (z, v):
        if t.shape != q_pre.shape or t.stride() != q_pre.stride() or t.dtype != q_pre.dtype:
            raise ValueError("q_pre, z, v must share shape, strides and dtype")
    if d_out.shape != q_pre.shape or d_out.dtype != q_pre.dtype:
        raise ValueError("d_out must have q_pre's shape and dtype")
    if norm_weight is not None and (norm_weight.dtype != torch.float32 or not norm_weight.is_contiguous()
                                    or norm_weight.numel() != Hh * d):
        raise ValueError("norm_weight must be contiguous fp32 [Hh, d]")
    if grads is None:
        grads = tuple(torch.empty_like(q_pre, dtype=grad_dtype or q_pre.dtype) for _ in range(3))
    dq, dz, dv = grads
    for t in grads:
        if t.shape != q_pre.shape or t.stride() != dq.stride() or t.dtype != dq.dtype:
            raise ValueError("gradient tensors must share q_pre's shape and one set of strides and dtype")
    if dweight is None and want_dweight:
        dweight = torch.empty((Hh, d), dtype=torch.float32, device=q_pre.device)
    if dweight is not None and (dweight.dtype != torch.float32 or not dweight.is_contiguous() or dweight.numel() != Hh * d):
        raise ValueError("dweight must be contiguous fp32 [Hh, d]")
    need = lasad_backward_layer_workspace_bytes(q_pre)
    if workspace is None and need:
        workspace = _scratch(need, q_pre.device, stream)
    li, lo, lg = _layout(q_pre), _layout(d_out), _layout(dq)
    _check(load().lasad_backward_layer(
        _ptr(q_pre), _ptr(z), _ptr(v), _ptr(d_out), _ptr(dq), _ptr(dz), _ptr(dv), _ptr(dweight),
        ctypes.byref(li), ctypes.byref(lo), ctypes.byref(lg), _dtype_code(q_pre), _dtype_code(dq),
        B, Hh, d, grid_h, grid_w, start_pos, n, boundary_mode, q_scale, _ptr(norm_weight), norm_eps,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return dq, dz, dv, dweight


def lasad_backward_layer_norm(q_pre: torch.Tensor, z: torch.Tensor, v: torch.Tensor, d_out: torch.Tensor,
                              grid_h: int, grid_w: int, norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                              start_pos: int = 0, boundary_mode: int = RESET_LAST_COL, q_scale: float = 1.0,
                              d_o: torch.Tensor | None = None, d_o_dtype: torch.dtype | None = None,
                              want_dweight: bool = True, workspace: torch.Tensor | None = None, stream=None):
    """The normalisation's part of lasad_backward_layer alone: returns (d_o, dweight), d_o = dL/d(recurrence
    output) in the inputs' dtype (or fp32 on request)."""
    B, n, Hh, d = q_pre.shape
    for t in (z, v):
        if t.shape != q_pre.shape or t.stride() != q_pre.stride() or t.dtype != q_pre.dtype:
            raise ValueError("q_pre, z, v must share shape, strides and dtype")
    if d_out.shape != q_pre.shape or d_out.dtype != q_pre.dtype:
        raise ValueError("d_out must have q_pre's shape and dtype")
    if d_o is None:
        d_o = torch.empty(q_pre.shape, dtype=d_o_dtype or q_pre.dtype, device=q_pre.device)
    if d_o.shape != q_pre.shape:
        raise ValueError("d_o must have q_pre's shape")
    dweight = torch.empty((Hh, d), dtype=torch.float32, device=q_pre.device) if want_dweight else None
    need = lasad_backward_layer_workspace_bytes(q_pre)
    if workspace is None and need:
        workspace = _scratch(need, q_pre.device, stream)
    li, lo, ld = _layout(q_pre), _layout(d_out), _layout(d_o)
    _check(load().lasad_backward_layer_norm(
        _ptr(q_pre), _ptr(z), _ptr(v), _ptr(d_out), _ptr(d_o), _ptr(dweight),
        ctypes.byref(li), ctypes.byref(lo), ctypes.byref(ld), _dtype_code(q_pre), _dtype_code(d_o),
        B, Hh, d, grid_h, grid_w, start_pos, n, boundary_mode, q_scale, _ptr(norm_weight), norm_eps,
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return d_o, dweight


# ---- the operators of a softmax layer: norms and rotation of query and key heads ----

def _rows(t: torch.Tensor, what: str) -> Layout:
    """Strides of a logical [B, n, heads, d] tensor; those of dimensions of size one, which torch may set to anything, are 0."""
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{what} must be [B, n_tokens, heads, d] with unit stride along d")
    if t.numel() == 0:
        return Layout(0, t.shape[2] * t.shape[3], t.shape[3])
    return Layout(*(t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)))


def _fit(*integers: int):
    """Integers go through ctypes as their low 32 bits; those that have more are refused."""
    for x in integers:
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{x} does not fit 32 bits")


def _head_weights(q_weight, k_weight, Hq: int, Hk: int, d: int) -> bool:
    """Checks the norm weights of query and key heads; whether they are one [d] for all heads."""
    shared = None
    for w, heads in ((q_weight, Hq), (k_weight, Hk)):
        if w is None:
            continue
        if w.dtype != torch.float32 or not w.is_contiguous() or tuple(w.shape) not in ((d,), (heads, d)):
            raise ValueError("norm weights must be contiguous fp32 [heads, d] or [d]")
        if shared is not None and shared != (w.dim() == 1):
            raise ValueError("one norm weight is shared by the heads and the other is not")
        shared = w.dim() == 1
    return bool(shared)


def _qk_pair(q, k, what: str):
    if q.dim() != k.dim() or q.shape[:-2] != k.shape[:-2] or q.shape[-1] != k.shape[-1] or q.dtype != k.dtype:
        raise ValueError(f"{what} must share a dtype and every dimension but the heads")


def _pair_out(given, q, k, dtype, what: str):
    """The two tensors of `given`, checked, or new ones like q and k."""
    if given is None:
        return tuple(torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device) for t in (q, k))
    a, b = given
    if a.shape != q.shape or b.shape != k.shape or a.dtype != b.dtype:
        raise ValueError(f"{what} must have the shapes of q and k and one dtype")
    return a, b


def lasad_forward_qk(q: torch.Tensor, k: torch.Tensor, grid_h: int, grid_w: int,
                     q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                     rope: int = ROPE_2D, pairing: int = PAIR_ADJACENT, rope_base: float = 10000.0, start_pos: int = 0,
                     out: tuple | None = None, out_dtype: torch.dtype | None = None, stream=None):
    """RMS norm of every query and key head, weight, rotation by raster position (see include/lasad.h).  q: [B, n, Hq, d],
    k: [B, n, Hk, d] views; weights fp32 [heads, d] or [d]; norm_eps < 0 switches the norm off.  Returns the two tensors;
    `out` may give them, (q, k) for in place."""
    if out is None and out_dtype is None and stream is None:
        done = _fast("forward_qk", q, k, grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, start_pos)
        if done is not None:
            return done
    _qk_pair(q, k, "q and k")
    lq, lk = _rows(q, "q"), _rows(k, "k")
    B, n, Hq, d = q.shape
    Hk = k.shape[2]
    _fit(B, n, Hq, Hk, d, grid_h, grid_w, start_pos, rope, pairing)
    shared = _head_weights(q_weight, k_weight, Hq, Hk, d)
    qo, ko = _pair_out(out, q, k, out_dtype, "out")
    lqo, lko = _rows(qo, "out"), _rows(ko, "out")
    _reachable(q, k, qo, ko, q_weight, k_weight)
    _check(load().lasad_forward_qk(
        _ptr(q), _ptr(k), _ptr(qo), _ptr(ko), ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(lqo), ctypes.byref(lko),
        _dtype_code(q), _dtype_code(qo), B, Hq, Hk, d, grid_h, grid_w, start_pos, n,
        _ptr(q_weight), _ptr(k_weight), shared, norm_eps, rope, pairing, rope_base, _stream(stream)))
    return qo, ko


def lasad_backward_qk_workspace_bytes(B: int, n_q_heads: int, n_k_heads: int, n_tokens: int, d: int, shared_weight: bool) -> int:
    _fit(B, n_q_heads, n_k_heads, n_tokens, d)
    return int(load().lasad_backward_qk_workspace_bytes(B, n_q_heads, n_k_heads, n_tokens, d, shared_weight))


def lasad_backward_qk(q: torch.Tensor, k: torch.Tensor, d_q: torch.Tensor, d_k: torch.Tensor, grid_h: int, grid_w: int,
                      q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                      rope: int = ROPE_2D, pairing: int = PAIR_ADJACENT, rope_base: float = 10000.0, start_pos: int = 0,
                      grads: tuple | None = None, grad_dtype: torch.dtype | None = None, want_dweight: bool = True,
                      workspace: torch.Tensor | None = None, stream=None):
    """Gradients of lasad_forward_qk; d_q, d_k: those of its outputs.  Returns (dq, dk, dq_weight, dk_weight); the weight
    gradients are fp32 like the weights (without a weight: [heads, d], at ones), None without a norm or with
    want_dweight=False."""
    if grads is None and grad_dtype is None and workspace is None and stream is None:
        done = _fast("backward_qk", q, k, grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, start_pos, d_q, d_k,
                     want_dweight)
        if done is not None:
            return done
    _qk_pair(q, k, "q and k")
    if d_q.shape != q.shape or d_k.shape != k.shape or d_q.dtype != q.dtype or d_k.dtype != q.dtype:
        raise ValueError("d_q and d_k must have the shapes and the dtype of q and k")
    layouts = [_rows(t, what) for t, what in ((q, "q"), (k, "k"), (d_q, "d_q"), (d_k, "d_k"))]
    B, n, Hq, d = q.shape
    Hk = k.shape[2]
    _fit(B, n, Hq, Hk, d, grid_h, grid_w, start_pos, rope, pairing)
    shared = _head_weights(q_weight, k_weight, Hq, Hk, d)
    dq, dk = _pair_out(grads, q, k, grad_dtype, "grads")
    layouts += [_rows(dq, "grads"), _rows(dk, "grads")]
    dwq = dwk = None
    if want_dweight and norm_eps >= 0:
        dwq, dwk = (torch.empty((d,) if shared else (heads, d), dtype=torch.float32, device=q.device) for heads in (Hq, Hk))
        if workspace is None:
            need = lasad_backward_qk_workspace_bytes(B, Hq, Hk, n, d, shared)
            if need:
                workspace = _scratch(need, q.device, stream)
    _reachable(q, k, d_q, d_k, dq, dk, q_weight, k_weight, workspace)
    _check(load().lasad_backward_qk(
        _ptr(q), _ptr(k), _ptr(d_q), _ptr(d_k), _ptr(dq), _ptr(dk), _ptr(dwq), _ptr(dwk), *(ctypes.byref(x) for x in layouts),
        _dtype_code(q), _dtype_code(dq), B, Hq, Hk, d, grid_h, grid_w, start_pos, n,
        _ptr(q_weight), _ptr(k_weight), shared, norm_eps, rope, pairing, rope_base,
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)))
    return dq, dk, dwq, dwk


def _step_position(pos, B: int):
    """pos as an integer, or as a position for every batch row."""
    if not isinstance(pos, torch.Tensor):
        return pos, None
    if pos.dtype != torch.int32 or pos.numel() != B or not pos.is_contiguous():
        raise ValueError("positions of batch rows must be contiguous int32 [B]")
    return 0, pos


def lasad_decode_step_qk(q: torch.Tensor, k: torch.Tensor, grid_h: int, grid_w: int, pos,
                         q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                         rope: int = ROPE_2D, pairing: int = PAIR_ADJACENT, rope_base: float = 10000.0,
                         out: tuple | None = None, out_dtype: torch.dtype | None = None, stream=None):
    """lasad_forward_qk for one token: q [B, Hq, d], k [B, Hk, d] contiguous; pos: an integer, or an int32 tensor [B] on the
    device with a position for every row (off the grid: inactive, nothing written)."""
    if out is None and out_dtype is None and stream is None:
        done = _fast("decode_step_qk", q, k, grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, pos)
        if done is not None:
            return done
    _qk_pair(q, k, "q and k")
    if q.dim() != 3 or not q.is_contiguous() or not k.is_contiguous():
        raise ValueError("q and k must be contiguous [B, heads, d]")
    B, Hq, d = q.shape
    Hk = k.shape[1]
    pos, pos_rows = _step_position(pos, B)
    _fit(B, Hq, Hk, d, grid_h, grid_w, pos, rope, pairing)
    shared = _head_weights(q_weight, k_weight, Hq, Hk, d)
    qo, ko = _pair_out(out, q, k, out_dtype, "out")
    if not qo.is_contiguous() or not ko.is_contiguous():
        raise ValueError("out must be contiguous")
    _reachable(q, k, qo, ko, q_weight, k_weight, pos_rows)
    _check(load().lasad_decode_step_qk(
        _ptr(q), _ptr(k), _ptr(qo), _ptr(ko), _dtype_code(q), _dtype_code(qo), B, Hq, Hk, d, grid_h, grid_w, pos, _ptr(pos_rows),
        _ptr(q_weight), _ptr(k_weight), shared, norm_eps, rope, pairing, rope_base, _stream(stream)))
    return qo, ko


# ---- attention with a window and sinks ----

def _scale(scale, q: torch.Tensor) -> float:
    return (q.shape[-1] or 1) ** -0.5 if scale is None else scale


def _window_inputs(q, k, v, kv_lens):
    """Checks the tensors of a forward or backward; their layouts."""
    lq, lk, lv = _rows(q, "q"), _rows(k, "k"), _rows(v, "v")
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[3] != q.shape[3] or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q must be [B, n, Hq, d], k and v [B, m, Hk, d], of one dtype")
    if kv_lens is not None and (kv_lens.dtype != torch.int32 or kv_lens.numel() != q.shape[0] or not kv_lens.is_contiguous()):
        raise ValueError("kv_lens must be contiguous int32 [B]")
    return lq, lk, lv


def lasad_forward_window(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, window: int, sinks: int = 0, start_pos: int = 0,
                         kv_lens: torch.Tensor | None = None, scale: float | None = None,
                         out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None, want_lse: bool = False, stream=None):
    """Softmax attention in which position p sees the positions p - window + 1 .. p and the first `sinks` (see include/lasad.h).
    q: [B, n, Hq, d], the tokens from start_pos on; k, v: [B, m, Hk, d], those from 0 on; kv_lens: valid keys of each batch row
    (int32 [B] on the device); scale: d ** -0.5 unless given.  Returns o, with want_lse (o, lse [B, Hq, n])."""
    if out is None and out_dtype is None and stream is None:
        done = _fast("forward_window", q, k, v, window, sinks, start_pos, kv_lens, _scale(scale, q), want_lse)
        if done is not None:
            return done if want_lse else done[0]
    lq, lk, lv = _window_inputs(q, k, v, kv_lens)
    B, n, Hq, d = q.shape
    _fit(*q.shape, *k.shape, window, sinks, start_pos)
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out has the wrong shape")
    lo = _rows(out, "out")
    lse = torch.empty((B, Hq, n), dtype=torch.float32, device=q.device) if want_lse else None
    _reachable(q, k, v, out, kv_lens)
    _check(load().lasad_forward_window(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(lv), ctypes.byref(lo),
        _dtype_code(q), _dtype_code(out), B, Hq, k.shape[2], d, start_pos, n, k.shape[1], window, sinks, _ptr(kv_lens),
        _scale(scale, q), _stream(stream)))
    return (out, lse) if want_lse else out


def lasad_backward_window_workspace_bytes(B: int, n_q_heads: int, n_k_heads: int, d: int, n_tokens: int, n_keys: int, window: int,
                                          sinks: int) -> int:
    _fit(B, n_q_heads, n_k_heads, d, n_tokens, n_keys, window, sinks)
    return int(load().lasad_backward_window_workspace_bytes(B, n_q_heads, n_k_heads, d, n_tokens, n_keys, window, sinks))


def lasad_backward_window(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor, d_o: torch.Tensor,
                          window: int, sinks: int = 0, start_pos: int = 0, kv_lens: torch.Tensor | None = None,
                          scale: float | None = None, grads: tuple | None = None, grad_dtype: torch.dtype | None = None,
                          workspace: torch.Tensor | None = None, stream=None):
    """Gradients of lasad_forward_window from what it returned (o in q's dtype, lse) and d_o.  Returns (dq, dk, dv); those of
    shared key heads are summed over their query heads."""
    if grads is None and grad_dtype is None and workspace is None and stream is None:
        done = _fast("backward_window", q, k, v, o, lse, d_o, window, sinks, start_pos, kv_lens,
                     _scale(scale, q))
        if done is not None:
            return done
    lq, lk, lv = _window_inputs(q, k, v, kv_lens)
    B, n, Hq, d = q.shape
    m, Hk = k.shape[1:3]
    _fit(*q.shape, *k.shape, window, sinks, start_pos)
    for t in (o, d_o):
        if t.shape != q.shape or t.dtype != q.dtype:
            raise ValueError("o and d_o must have q's shape and dtype")
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, Hq, n) or not lse.is_contiguous():
        raise ValueError("lse must be contiguous fp32 [B, Hq, n]")
    if grads is None:
        grads = tuple(torch.empty(t.shape, dtype=grad_dtype or q.dtype, device=q.device) for t in (q, k, v))
    for t, x in zip(grads, (q, k, v)):
        if t.shape != x.shape or t.dtype != grads[0].dtype:
            raise ValueError("grads must have the shapes of q, k, v and one dtype")
    dq, dk, dv = grads
    layouts = [lq, lk, lv, _rows(o, "o"), _rows(d_o, "d_o"), _rows(dq, "grads"), _rows(dk, "grads"), _rows(dv, "grads")]
    if workspace is None:
        need = lasad_backward_window_workspace_bytes(B, Hq, Hk, d, n, m, window, sinks)
        if need:
            workspace = _scratch(need, q.device, stream)
    _reachable(q, k, v, o, lse, d_o, dq, dk, dv, kv_lens, workspace)
    _check(load().lasad_backward_window(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), *(ctypes.byref(x) for x in layouts),
        _dtype_code(q), _dtype_code(dq), B, Hq, Hk, d, start_pos, n, m, window, sinks, _ptr(kv_lens),
        _scale(scale, q),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)))
    return dq, dk, dv


def lasad_decode_step_window_workspace_bytes(B: int, n_q_heads: int, n_k_heads: int, d: int, cache_tokens: int, window: int,
                                             sinks: int) -> int:
    _fit(B, n_q_heads, n_k_heads, d, cache_tokens, window, sinks)
    return int(load().lasad_decode_step_window_workspace_bytes(B, n_q_heads, n_k_heads, d, cache_tokens, window, sinks))


def lasad_decode_step_window(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                             pos, window: int, sinks: int = 0, scale: float | None = None,
                             out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                             workspace: torch.Tensor | None = None, use_workspace: bool = True, stream=None) -> torch.Tensor:
    """lasad_forward_window for one token: q [B, Hq, d], k, v [B, Hk, d]; caches [B, Hk, rows, d], in which this call writes
    k and v to the token's row (key j: row j < sinks ? j : sinks + (j - sinks) % (rows - sinks)); pos: an integer, or an int32
    tensor [B] on the device (a row whose position does not fit the cache is inactive)."""
    if out is None and out_dtype is None and workspace is None and use_workspace and stream is None:
        done = _fast("decode_step_window", q, k, v, k_cache, v_cache, pos, window, sinks, _scale(scale, q))
        if done is not None:
            return done[0]
    B, Hq, d = q.shape
    _same(k, (v,), "k and v must be contiguous [B, Hk, d] of one shape and dtype")
    if not q.is_contiguous() or k.dim() != 3 or k.shape[0] != B or k.shape[2] != d or k.dtype != q.dtype:
        raise ValueError("q must be contiguous [B, Hq, d], k and v [B, Hk, d], of one dtype")
    Hk = k.shape[1]
    _same(k_cache, (v_cache,), "the caches must be contiguous, of one shape and dtype")
    if k_cache.dim() != 4 or k_cache.shape[:2] != (B, Hk) or k_cache.shape[3] != d or k_cache.dtype != q.dtype:
        raise ValueError("the caches must be [B, Hk, rows, d] in q's dtype")
    rows = k_cache.shape[2]
    pos, pos_rows = _step_position(pos, B)
    _fit(*q.shape, Hk, rows, pos, window, sinks)
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hq, d]")
    if workspace is None and use_workspace:
        need = lasad_decode_step_window_workspace_bytes(B, Hq, Hk, d, rows, window, sinks)
        if need:
            workspace = _scratch(need, q.device, stream)
    _reachable(q, k, v, k_cache, v_cache, out, pos_rows, workspace)
    _check(load().lasad_decode_step_window(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(k_cache), _ptr(v_cache), rows, _dtype_code(q), _dtype_code(out), B, Hq, Hk, d,
        pos, _ptr(pos_rows), window, sinks, _scale(scale, q),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


# ---- a cache in pages, held in 8 bits ----

PAGE = 64                              # positions of a page


class Pages(NamedTuple):
    """A pool of pages (see include/lasad.h): k [n_pages, Hk, 64, d] and v [n_pages, Hk, d, 64] of e4m3 codes, fp32 scales [n_pages, Hk]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor


def new_pages(n_pages: int, n_k_heads: int, d: int, device="cuda") -> Pages:
    """A pool of empty pages."""
    codes = [torch.empty(shape, dtype=torch.float8_e4m3fn, device=device) for shape in ((n_pages, n_k_heads, PAGE, d), (n_pages, n_k_heads, d, PAGE))]
    return Pages(*codes, *(torch.empty((n_pages, n_k_heads), dtype=torch.float32, device=device) for _ in range(2)))


def _pages(pages, table, Hk: int, d: int, B: int) -> PagesStruct:
    k, v, k_scales, v_scales = pages
    n = k.shape[0]
    for t, shape in ((k, (n, Hk, PAGE, d)), (v, (n, Hk, d, PAGE))):
        if tuple(t.shape) != shape or t.dtype != torch.float8_e4m3fn or not t.is_contiguous():
            raise ValueError("the pages must be contiguous float8_e4m3fn, [n_pages, Hk, 64, d] of k and [n_pages, Hk, d, 64] of v")
    for t in (k_scales, v_scales):
        if tuple(t.shape) != (n, Hk) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("the scales must be contiguous fp32 [n_pages, Hk]")
    if table.dim() != 2 or table.shape[0] != B or table.dtype != torch.int32 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("the table must be int32 [B, pages] with unit stride along the pages")
    _fit(n, table.shape[1])
    _reachable(k, v, k_scales, v_scales, table)
    return PagesStruct(_ptr(k), _ptr(v), _ptr(k_scales), _ptr(v_scales), n, table.shape[1], _ptr(table), table.stride(0) if B > 1 else 0)


def _packed(t: torch.Tensor, what: str) -> Layout:
    """Strides of packed tokens [T, heads, d]."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what} must be [tokens, heads, d] with unit stride along d")
    if t.numel() == 0:
        return Layout(0, t.shape[1] * t.shape[2], t.shape[2])
    return Layout(0, *(t.stride(i) if t.shape[i] > 1 else 0 for i in range(2)))


def _row_starts(row_starts, B: int):
    if row_starts is not None and (row_starts.dtype != torch.int32 or tuple(row_starts.shape) != (B + 1,) or not row_starts.is_contiguous()):
        raise ValueError("row_starts must be contiguous int32 [B + 1]")


def lasad_append_pages(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, pages: Pages, table: torch.Tensor, pos,
                       grid_h: int, grid_w: int, q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                       norm_eps: float = 1e-6, rope: int = ROPE_2D, pairing: int = PAIR_ADJACENT, rope_base: float = 10000.0,
                       row_starts: torch.Tensor | None = None, out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                       stream=None):
    """Appends the new tokens of the table's rows to their pages (see include/lasad.h), keys normed and rotated by raster position as in
    lasad_forward_qk.  q [T, Hq, d], k, v [T, Hk, d]: views of packed tokens; row_starts: int32 [B + 1] on the device, None: one token a row;
    pos: position of the rows' first new token, an integer or an int32 tensor [B] on the device (off the grid or the table: inactive); table:
    int32 [B, pages].  Returns the normed and rotated queries (None without q); `out` may give them, q itself for in place."""
    if q is not None and out is None and out_dtype is None and stream is None:
        done = _fast("append_pages", q, k, v, pages, table, pos, grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, row_starts)
        if done is not None:
            return done[0]
    if k.shape != v.shape or k.dtype != v.dtype:
        raise ValueError("k and v must have one shape and dtype")
    lk, lv = _packed(k, "k"), _packed(v, "v")
    T, Hk, d = k.shape
    B = table.shape[0]
    p = _pages(pages, table, Hk, d, B)
    _row_starts(row_starts, B)
    pos, pos_rows = _step_position(pos, B)
    Hq, lq, lo = 0, None, None
    if q is None:
        if out is not None or q_weight is not None:
            raise ValueError("out or q_weight without q")
    else:
        lq = _packed(q, "q")
        Hq = q.shape[1]
        if q.shape[0] != T or q.shape[2] != d or q.dtype != k.dtype:
            raise ValueError("q must share a dtype and every dimension but the heads with k")
        if out is None:
            out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        elif out.shape != q.shape:
            raise ValueError("out has the wrong shape")
        lo = _packed(out, "out")
    _fit(T, Hq, Hk, d, B, grid_h, grid_w, pos, rope, pairing)
    shared = _head_weights(q_weight, k_weight, Hq, Hk, d)
    _reachable(q, k, v, out, q_weight, k_weight, row_starts, pos_rows)
    _check(load().lasad_append_pages(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), lq and ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(lv), lo and ctypes.byref(lo), ctypes.byref(p),
        _dtype_code(k), _dtype_code(k if out is None else out), B, Hq, Hk, d, grid_h, grid_w, T, _ptr(row_starts), pos, _ptr(pos_rows),
        _ptr(q_weight), _ptr(k_weight), shared, norm_eps, rope, pairing, rope_base, _stream(stream)))
    return out


def lasad_forward_pages_workspace_bytes(B: int, n_q_heads: int, n_k_heads: int, d: int, n_tokens: int, one_each: bool, table_pages: int,
                                        window: int, sinks: int) -> int:
    _fit(B, n_q_heads, n_k_heads, d, n_tokens, table_pages, window, sinks)
    return int(load().lasad_forward_pages_workspace_bytes(B, n_q_heads, n_k_heads, d, n_tokens, bool(one_each), table_pages, window, sinks))


def lasad_forward_pages(q: torch.Tensor, pages: Pages, table: torch.Tensor, pos, window: int, sinks: int = 0,
                        row_starts: torch.Tensor | None = None, scale: float | None = None,
                        out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                        workspace: torch.Tensor | None = None, use_workspace: bool = True, stream=None) -> torch.Tensor:
    """lasad_forward_window of packed queries [T, Hq, d] (normed and rotated, their keys appended) over the rows' pages; rows, positions and
    table as in lasad_append_pages.  Queries of inactive rows (a position that is negative or behind the table; no grid is known here) and of
    none are left as they were in `out`."""
    if out is None and out_dtype is None and workspace is None and use_workspace and stream is None:
        done = _fast("forward_pages", q, pages, table, pos, window, sinks, row_starts, _scale(scale, q))
        if done is not None:
            return done[0]
    lq = _packed(q, "q")
    T, Hq, d = q.shape
    B, Hk = table.shape[0], pages[0].shape[1]
    p = _pages(pages, table, Hk, d, B)
    _row_starts(row_starts, B)
    pos, pos_rows = _step_position(pos, B)
    _fit(T, Hq, Hk, d, B, pos, window, sinks)
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out has the wrong shape")
    lo = _packed(out, "out")
    if workspace is None and use_workspace:
        need = lasad_forward_pages_workspace_bytes(B, Hq, Hk, d, T, row_starts is None, table.shape[1], window, sinks)
        if need:
            workspace = _scratch(need, q.device, stream)
    _reachable(q, out, row_starts, pos_rows, workspace)
    _check(load().lasad_forward_pages(
        _ptr(q), _ptr(out), ctypes.byref(lq), ctypes.byref(lo), ctypes.byref(p), _dtype_code(q), _dtype_code(out), B, Hq, Hk, d, T,
        _ptr(row_starts), pos, _ptr(pos_rows), window, sinks, _scale(scale, q),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


def lasad_decode_step_pages_workspace_bytes(B: int, n_q_heads: int, n_k_heads: int, d: int, table_pages: int, window: int, sinks: int) -> int:
    _fit(B, n_q_heads, n_k_heads, d, table_pages, window, sinks)
    return int(load().lasad_decode_step_pages_workspace_bytes(B, n_q_heads, n_k_heads, d, table_pages, window, sinks))


def lasad_decode_step_pages(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, pages: Pages, table: torch.Tensor, pos,
                            grid_h: int, grid_w: int, window: int, sinks: int = 0,
                            q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, norm_eps: float = 1e-6,
                            rope: int = ROPE_2D, pairing: int = PAIR_ADJACENT, rope_base: float = 10000.0, scale: float | None = None,
                            out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                            workspace: torch.Tensor | None = None, use_workspace: bool = True, stream=None) -> torch.Tensor:
    """One token of every row: q [B, Hq, d], k, v [B, Hk, d] contiguous, as they leave the projection; norms, rotation, append to the
    pages and attention over them.  pos and table as in lasad_append_pages; an inactive row's output is not written."""
    if out is None and out_dtype is None and workspace is None and use_workspace and stream is None:
        done = _fast("decode_step_pages", q, k, v, pages, table, pos, grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base,
                     window, sinks, _scale(scale, q))
        if done is not None:
            return done[0]
    B, Hq, d = q.shape
    _same(k, (v,), "k and v must be contiguous [B, Hk, d] of one shape and dtype")
    if not q.is_contiguous() or k.dim() != 3 or k.shape[0] != B or k.shape[2] != d or k.dtype != q.dtype:
        raise ValueError("q must be contiguous [B, Hq, d], k and v [B, Hk, d], of one dtype")
    Hk = k.shape[1]
    p = _pages(pages, table, Hk, d, B)
    pos, pos_rows = _step_position(pos, B)
    _fit(*q.shape, Hk, grid_h, grid_w, pos, rope, pairing, window, sinks)
    shared = _head_weights(q_weight, k_weight, Hq, Hk, d)
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be contiguous [B, Hq, d]")
    if workspace is None and use_workspace:
        need = lasad_decode_step_pages_workspace_bytes(B, Hq, Hk, d, table.shape[1], window, sinks)
        if need:
            workspace = _scratch(need, q.device, stream)
    _reachable(q, k, v, out, q_weight, k_weight, pos_rows, workspace)
    _check(load().lasad_decode_step_pages(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), ctypes.byref(p), _dtype_code(q), _dtype_code(out), B, Hq, Hk, d, grid_h, grid_w, pos, _ptr(pos_rows),
        _ptr(q_weight), _ptr(k_weight), shared, norm_eps, rope, pairing, rope_base, window, sinks, _scale(scale, q),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


# ---- host <-> device helpers for seeded numpy inputs (no arithmetic) ---------

def to_device(x, dtype: str, device="cuda"):
    """Upload a float32 numpy array (values already storage-rounded) as an f32 or bf16 tensor,
    keeping the numpy array's strides (so a transposed view stays a transposed view)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(x))
    if not x.flags.c_contiguous:
        # rebuild the same permutation on the device
        order = sorted(range(x.ndim), key=lambda i: -x.strides[i])
        t = torch.from_numpy(np.ascontiguousarray(x.transpose(order)))
        inv = [order.index(i) for i in range(x.ndim)]
        t = t.to(device).permute(inv)
    else:
        t = t.to(device)
    if dtype == "bf16":
        return t.to(torch.bfloat16)    # exact: the values are already bf16-representable
    if dtype == "f32":
        return t
    raise ValueError(dtype)
