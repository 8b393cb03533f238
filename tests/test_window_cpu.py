"""Attention with a window and sinks without a GPU: the reference itself, and what the C ABI and the binding refuse."""
import ctypes

import pytest
import torch

import softmax_layer_reference as ref
from paper_2507_01652_amd import binding

L = binding.Layout


def test_the_reference_against_differences_and_automatic_differentiation():
    B, n, m, Hq, Hk, d = 2, 5, 7, 4, 2, 4
    q, k, v = (ref.draw(s, torch.float64, i).requires_grad_() for i, s in enumerate(((B, n, Hq, d), (B, m, Hk, d), (B, m, Hk, d))))
    mask = ref.seen_mask(n, m, 3, 3, 1, [7, 2], B)
    assert not mask[1].any(-1).any(0).all() or mask.any()
    fn = lambda a, b, c: ref.window_forward(a, b, c, mask, 0.5)[0]
    assert torch.autograd.gradcheck(fn, (q, k, v))
    do = ref.draw(q.shape, torch.float64, 9)
    fn(q, k, v).backward(do)
    with torch.no_grad():
        for got, x in zip(ref.window_backward(q, k, v, do, mask, 0.5), (q, k, v)):
            assert torch.allclose(got, x.grad, rtol=1e-12, atol=1e-14)


def test_the_mask_by_hand():
    seen = ref.seen_mask(4, 9, 4, 2, 1, [6], 1)[0].int().tolist()
    assert seen == [[1, 0, 0, 1, 1, 0, 0, 0, 0], [1, 0, 0, 0, 1, 1, 0, 0, 0], [1, 0, 0, 0, 0, 1, 0, 0, 0], [1, 0, 0, 0, 0, 0, 0, 0, 0]]


def _forward(**kw):
    a = dict(q=0x1000, k=0x2000, v=0x3000, o=0x4000, lse=0x5000, lq=L(1024, 256, 64), lk=L(512, 128, 64), lv=L(512, 128, 64),
             lo=L(1024, 256, 64), io=1, ot=1, B=1, Hq=4, Hk=2, d=64, start=0, n=4, m=4, window=2, sinks=1, lens=None, scale=0.125)
    a.update(kw)
    by = lambda x: None if x is None else ctypes.byref(x)
    return binding.load().lasad_forward_window(a["q"], a["k"], a["v"], a["o"], a["lse"], by(a["lq"]), by(a["lk"]), by(a["lv"]), by(a["lo"]),
                                               a["io"], a["ot"], a["B"], a["Hq"], a["Hk"], a["d"], a["start"], a["n"], a["m"], a["window"],
                                               a["sinks"], a["lens"], a["scale"], None)


BAD = [dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=0x1008), dict(o=0x4004), dict(lse=0x5002), dict(lens=0x6001),
       dict(lq=None), dict(lk=None), dict(lv=None), dict(lo=None), dict(lq=L(1024, 254, 64)), dict(lv=L(512, -128, 64)), dict(lo=L(1024, 0, 64)),
       dict(lo=L(1024, 256, 32)), dict(io=2), dict(ot=7), dict(io=0, ot=1), dict(B=0), dict(Hq=0), dict(Hk=0), dict(Hq=3), dict(d=96),
       dict(n=-1), dict(m=-1), dict(start=-1), dict(start=1 << 30), dict(m=(1 << 30) + 1), dict(window=0), dict(window=-5), dict(sinks=-1),
       dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(o=0x1000), dict(o=0x3000), dict(lse=0x4000),
       dict(B=1 << 22, n=1 << 10), dict(B=1 << 16, Hq=1 << 14, Hk=1)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: ",".join(b))
def test_refused_before_a_launch(bad):
    assert _forward(**bad) in (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)
    assert len(binding.load().lasad_last_error()) > 4


def test_no_tokens_is_no_launch():
    assert _forward(n=0, q=None, o=None, lse=None) == binding.OK


def _backward(**kw):
    a = dict(q=0x1000, k=0x2000, v=0x3000, o=0x4000, lse=0x5000, do=0x6000, dq=0x7000, dk=0x8000, dv=0x9000, ws=0xa000, size=1 << 20, m=4, n=4,
             ldk=L(512, 128, 64), io=1, gt=1)
    a.update(kw)
    by = ctypes.byref
    lq, lk = L(1024, 256, 64), L(512, 128, 64)
    return binding.load().lasad_backward_window(a["q"], a["k"], a["v"], a["o"], a["lse"], a["do"], a["dq"], a["dk"], a["dv"], by(lq), by(lk),
                                                by(lk), by(lq), by(lq), by(lq), by(a["ldk"]), by(lk), a["io"], a["gt"], 1, 4, 2, 64, 0, a["n"], a["m"],
                                                2, 1, None, 0.125, a["ws"], a["size"], None)


@pytest.mark.parametrize("bad", [dict(lse=None), dict(do=None), dict(dq=None), dict(dk=None), dict(dv=0x9008), dict(dq=0x1000), dict(dk=0x3000),
                                 dict(dv=0x8000), dict(dq=0x6000), dict(ldk=L(512, 64, 64), gt=0, io=0, dk=0x8004), dict(ldk=L(512, 0, 64)),
                                 dict(io=0, gt=1), dict(ws=0xa008)], ids=lambda b: ",".join(b))
def test_the_backward_refuses(bad):
    assert _backward(**bad) in (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)


def test_the_backward_needs_its_workspace():
    need = binding.lasad_backward_window_workspace_bytes(1, 4, 2, 64, 4, 4, 2, 1)
    assert need >= 4 * 4 * 4
    assert _backward(ws=None) == binding.ERR_WORKSPACE
    assert _backward(size=need - 1) == binding.ERR_WORKSPACE
    # long sequences: the sinks' tile in parts; never more than 1024 of them, whatever the sizes
    more = binding.lasad_backward_window_workspace_bytes(1, 4, 2, 64, 4096, 4096, 64, 1)
    assert more > binding.lasad_backward_window_workspace_bytes(1, 4, 2, 64, 4096, 4096, 64, 0)
    assert binding.lasad_backward_window_workspace_bytes(64, 16, 16, 128, 1 << 16, 1 << 16, 16, 1 << 16) <= 64 * 16 * (1 << 16) * 4 + 256


def _step(**kw):
    a = dict(q=0x1000, k=0x2000, v=0x3000, o=0x4000, kc=0x10000, vc=0x20000, cap=8, io=1, ot=1, B=2, Hq=4, Hk=2, d=64, pos=3, rows=None,
             window=4, sinks=2, scale=0.125, ws=None, size=0)
    a.update(kw)
    return binding.load().lasad_decode_step_window(a["q"], a["k"], a["v"], a["o"], a["kc"], a["vc"], a["cap"], a["io"], a["ot"], a["B"], a["Hq"],
                                                   a["Hk"], a["d"], a["pos"], a["rows"], a["window"], a["sinks"], a["scale"], a["ws"], a["size"], None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(kc=None), dict(vc=0x20008), dict(o=0x4008), dict(cap=2), dict(cap=0), dict(pos=-1),
                                 dict(pos=8, window=7), dict(pos=8, cap=5, window=4), dict(window=0), dict(sinks=-1), dict(scale=0.0), dict(Hq=5),
                                 dict(d=16), dict(B=0), dict(io=0, ot=1), dict(rows=0x7002), dict(o=0x1000), dict(kc=0x20000), dict(k=0x10000),
                                 dict(o=0x10000), dict(ws=0x30008, size=1 << 20)], ids=lambda b: ",".join(b))
def test_the_step_refuses(bad):
    assert _step(**bad) in (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)


def test_a_step_workspace_that_is_too_small_is_refused():
    size = lambda **k: binding.lasad_decode_step_window_workspace_bytes(*{**dict(B=1, Hq=4, Hk=2, d=64, cap=9000, window=8000, sinks=4), **k}.values())
    need = size()
    assert need > 0 and size(B=4096) == 0 and size(window=100) == 0 and size(cap=100) == 0
    assert _step(B=1, cap=9000, window=8000, sinks=4, ws=0x30000, size=need - 1) == binding.ERR_WORKSPACE


Q, K = torch.zeros(2, 5, 4, 64), torch.zeros(2, 7, 2, 64)


@pytest.mark.parametrize("change", [
    dict(k=torch.zeros(3, 7, 2, 64)), dict(v=torch.zeros(2, 6, 2, 64)), dict(k=K.bfloat16()), dict(q=torch.zeros(2, 5, 4, 128)[..., ::2]),
    dict(kv_lens=torch.zeros(2)), dict(kv_lens=torch.zeros(3, dtype=torch.int32)), dict(out=torch.zeros(2, 5, 2, 64)), dict(),
], ids=lambda c: ",".join(c) or "host memory")
def test_the_binding_refuses(change):
    a = dict(q=Q, k=K, v=K)
    a.update(change)
    with pytest.raises(ValueError):
        binding.lasad_forward_window(a.pop("q"), a.pop("k"), a.pop("v"), 4, **a)


@pytest.mark.parametrize("change", [
    dict(o=K), dict(d_o=Q.bfloat16()), dict(lse=torch.zeros(2, 5, 4)), dict(lse=torch.zeros(2, 4, 5).double()), dict(grads=(Q, K, Q)), dict(),
], ids=lambda c: ",".join(c) or "host memory")
def test_the_binding_refuses_backwards(change):
    a = dict(o=Q, lse=torch.zeros(2, 4, 5), d_o=Q)
    a.update(change)
    with pytest.raises(ValueError):
        binding.lasad_backward_window(Q, K, K, a.pop("o"), a.pop("lse"), a.pop("d_o"), 4, **a)


@pytest.mark.parametrize("change", [
    dict(q=torch.zeros(2, 4, 128)[..., ::2]), dict(k=torch.zeros(2, 2, 32)), dict(v=torch.zeros(2, 3, 64)), dict(k_cache=torch.zeros(2, 2, 9, 32)),
    dict(v_cache=torch.zeros(2, 2, 8, 64)), dict(k_cache=torch.zeros(2, 9, 2, 64).transpose(1, 2)), dict(pos=torch.zeros(2)),
    dict(out=torch.zeros(2, 2, 64)), dict(),
], ids=lambda c: ",".join(c) or "host memory")
def test_the_binding_refuses_steps(change):
    a = dict(q=torch.zeros(2, 4, 64), k=torch.zeros(2, 2, 64), v=torch.zeros(2, 2, 64), k_cache=torch.zeros(2, 2, 9, 64),
             v_cache=torch.zeros(2, 2, 9, 64), pos=0)
    a.update(change)
    with pytest.raises(ValueError):
        binding.lasad_decode_step_window(a["q"], a["k"], a["v"], a["k_cache"], a["v_cache"], a["pos"], 4, out=a.get("out"))
