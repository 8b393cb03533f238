"""Head norms with raster rotation without a GPU: the reference itself, and what the C ABI and the binding refuse."""
import ctypes

import pytest
import torch

import softmax_layer_reference as ref
from paper_2507_01652_amd import binding


@pytest.mark.parametrize("rope,halves,w", [(0, False, True), (1, False, True), (1, True, False), (2, False, True), (2, True, True)])
def test_the_reference_against_differences(rope, halves, w):
    d = 8
    x = ref.draw((2, 3, 2, d), torch.float64, 1).requires_grad_()
    wt = (ref.draw((2, d), torch.float64, 2, 0.3) + 1).requires_grad_() if w else None
    pos = torch.tensor([[4, 5, 6], [11, 12, 13]])
    assert torch.autograd.gradcheck(lambda a, b: ref.qk_row(a, b, pos, 5, rope, halves, 100.0, 1e-3), (x, wt))


@pytest.mark.parametrize("halves", [False, True])
def test_the_rotation_keeps_sizes_and_turns_relative_positions(halves):
    d = 16
    q, k = ref.draw((1, 1, d), torch.float64, 3), ref.draw((1, 1, d), torch.float64, 4)
    turn = lambda x, p, rope: ref.qk_row(x, None, torch.tensor([p]), 7, rope, halves, 10000.0, -1.0)
    assert torch.allclose(turn(q, 13, 2).norm(), q.norm())
    dots = [float((turn(q, p + 5, 1) * turn(k, p, 1)).sum()) for p in (0, 9, 1000)]
    assert max(dots) - min(dots) < 1e-9
    dots = [float((turn(q, (r + 2) * 7 + c + 1, 2) * turn(k, r * 7 + c, 2)).sum()) for r, c in ((0, 0), (3, 5), (90, 2))]
    assert max(dots) - min(dots) < 1e-9
    assert torch.equal(turn(q, 0, 2), q)
    # two axes: a row further turns the first half of the channels and nothing else
    a, b = turn(q, 3, 2), turn(q, 3 + 7, 2)
    moved = (a != b).flatten()
    assert moved[: d // 2].all() and not moved[d // 2:].any()


L = binding.Layout


def _forward(**kw):
    a = dict(q=0x1000, k=0x2000, qo=0x3000, ko=0x4000, lq=L(1024, 256, 64), lk=L(512, 128, 64), lqo=L(1024, 256, 64), lko=L(512, 128, 64),
             io=1, ot=1, B=1, Hq=4, Hk=2, d=64, gh=2, gw=2, start=0, n=4, wq=None, wk=None, shared=0, eps=1e-6, rope=2, pairing=0,
             base=10000.0)
    a.update(kw)
    ref_ = lambda x: None if x is None else ctypes.byref(x)
    return binding.load().lasad_forward_qk(a["q"], a["k"], a["qo"], a["ko"], ref_(a["lq"]), ref_(a["lk"]), ref_(a["lqo"]), ref_(a["lko"]),
                                           a["io"], a["ot"], a["B"], a["Hq"], a["Hk"], a["d"], a["gh"], a["gw"], a["start"], a["n"],
                                           a["wq"], a["wk"], a["shared"], a["eps"], a["rope"], a["pairing"], a["base"], None)


BAD = [dict(q=None), dict(ko=None), dict(q=0x1008), dict(lq=None), dict(lqo=None), dict(lq=L(1024, 252, 64)), dict(lk=L(512, -128, 64)),
       dict(lqo=L(1024, 0, 64)), dict(lqo=L(1024, 256, 32)), dict(lko=L(0, 128, 64), B=2), dict(io=2), dict(ot=-1), dict(io=0, ot=1),
       dict(B=0), dict(Hq=0), dict(Hk=-1), dict(d=48), dict(n=-1), dict(n=5), dict(start=-1), dict(start=1), dict(gh=0), dict(gw=0),
       dict(gh=1 << 16, gw=1 << 15), dict(rope=3), dict(rope=-1), dict(pairing=2), dict(base=1.0), dict(base=float("nan")),
       dict(base=float("inf")), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0, wq=0x5000), dict(wk=0x5004),
       dict(qo=0x1000, ot=0), dict(qo=0x1000, lqo=L(2048, 512, 64)), dict(qo=0x2000), dict(ko=0x1000), dict(qo=0x4000),
       dict(B=1 << 20, n=1 << 12, gh=1 << 10, gw=1 << 10)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: ",".join(b))
def test_refused_before_a_launch(bad):
    assert _forward(**bad) in (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)
    assert len(binding.load().lasad_last_error()) > 4


def test_no_tokens_is_no_launch():
    assert _forward(n=0, q=None, k=None, qo=None, ko=None) == binding.OK


def test_the_backward_needs_its_workspace():
    lib = binding.load()
    need = binding.lasad_backward_qk_workspace_bytes(1, 4, 2, 4, 64, False)
    assert need >= 6 * 64 * 4
    lq, lk = L(1024, 256, 64), L(512, 128, 64)
    by = ctypes.byref

    def call(dwq=0x9000, ws=0xa000, size=need, dq=0x5000, eps=1e-6):
        return lib.lasad_backward_qk(0x1000, 0x2000, 0x3000, 0x4000, dq, 0x6000, dwq, None, by(lq), by(lk), by(lq), by(lk), by(lq), by(lk),
                                     1, 1, 1, 4, 2, 64, 2, 2, 0, 4, None, None, 0, eps, 2, 0, 10000.0, ws, size, None)
    assert call(ws=None) == binding.ERR_WORKSPACE
    assert call(size=need - 1) == binding.ERR_WORKSPACE
    assert call(ws=0xa004) == binding.ERR_INVALID_ARG
    assert call(dq=0x1000) == binding.ERR_INVALID_ARG
    assert call(eps=-1.0) == binding.ERR_INVALID_ARG


Q, K = torch.zeros(2, 5, 4, 64), torch.zeros(2, 5, 2, 64)


@pytest.mark.parametrize("change", [
    dict(k=torch.zeros(2, 4, 2, 64)), dict(k=torch.zeros(2, 5, 2, 32)), dict(k=K.bfloat16()), dict(q=torch.zeros(2, 5, 4, 128)[..., ::2]),
    dict(q_weight=torch.ones(2, 64)), dict(q_weight=torch.ones(64).double()), dict(q_weight=torch.ones(64), k_weight=torch.ones(2, 64)),
    dict(k_weight=torch.ones(128)[::2]), dict(out=(Q, Q)), dict(out=(Q, K.bfloat16())), dict(),
], ids=lambda c: ",".join(c) or "host memory")
def test_the_binding_refuses(change):
    a = dict(q=Q, k=K)
    a.update(change)
    with pytest.raises(ValueError):
        binding.lasad_forward_qk(a.pop("q"), a.pop("k"), 4, 4, **a)


@pytest.mark.parametrize("change", [
    dict(q=torch.zeros(2, 4, 128)[..., ::2]), dict(pos=torch.zeros(2)), dict(pos=torch.zeros(3, dtype=torch.int32)), dict(),
], ids=lambda c: ",".join(c) or "host memory")
def test_the_binding_refuses_steps(change):
    a = dict(q=torch.zeros(2, 4, 64), k=torch.zeros(2, 2, 64), pos=0)
    a.update(change)
    with pytest.raises(ValueError):
        binding.lasad_decode_step_qk(a["q"], a["k"], 4, 4, a["pos"])
