"""The paged 8-bit cache without a GPU: what the C ABI and the binding refuse, size queries, the reference's own parts."""
import ctypes

import pytest
import torch

import pages_reference as pr
from paper_2507_01652_amd import binding

L = binding.Layout


def _struct(**kw):
    a = dict(k=0x10000, v=0x20000, ks=0x30000, vs=0x40000, n=8, pages=4, table=0x50000, stride=4)
    a.update(kw)
    return binding.PagesStruct(a["k"], a["v"], a["ks"], a["vs"], a["n"], a["pages"], a["table"], a["stride"])


def _by(x):
    return None if x is None else ctypes.byref(x)


def _append(pages=_struct(), **kw):
    a = dict(q=0x1000, k=0x2000, v=0x3000, out=0x4000, lq=L(0, 256, 64), lk=L(0, 128, 64), lv=L(0, 128, 64), lo=L(0, 256, 64), io=1, ot=1, B=2, Hq=4, Hk=2,
             d=64, gh=16, gw=16, n=5, starts=0x5000, pos=0, rows=None, wq=None, wk=None, shared=0, eps=1e-6, rope=2, pair=0, base=1e4)
    a.update(kw)
    return binding.load().lasad_append_pages(a["q"], a["k"], a["v"], a["out"], _by(a["lq"]), _by(a["lk"]), _by(a["lv"]), _by(a["lo"]), _by(pages), a["io"],
                                             a["ot"], a["B"], a["Hq"], a["Hk"], a["d"], a["gh"], a["gw"], a["n"], a["starts"], a["pos"], a["rows"],
                                             a["wq"], a["wk"], a["shared"], a["eps"], a["rope"], a["pair"], a["base"], None)


def _forward(pages=_struct(), **kw):
    a = dict(q=0x1000, o=0x4000, lq=L(0, 256, 64), lo=L(0, 256, 64), io=1, ot=1, B=2, Hq=4, Hk=2, d=64, n=5, starts=0x5000, pos=0, rows=None, window=7,
             sinks=1, scale=0.125, ws=None, bytes=0)
    a.update(kw)
    return binding.load().lasad_forward_pages(a["q"], a["o"], _by(a["lq"]), _by(a["lo"]), _by(pages), a["io"], a["ot"], a["B"], a["Hq"], a["Hk"], a["d"],
                                              a["n"], a["starts"], a["pos"], a["rows"], a["window"], a["sinks"], a["scale"], a["ws"], a["bytes"], None)


def _step(pages=_struct(), **kw):
    a = dict(q=0x1000, k=0x2000, v=0x3000, o=0x4000, io=1, ot=1, B=2, Hq=4, Hk=2, d=64, gh=16, gw=16, pos=0, rows=None, wq=None, wk=None, shared=0, eps=1e-6,
             rope=2, pair=0, base=1e4, window=7, sinks=1, scale=0.125, ws=None, bytes=0)
    a.update(kw)
    return binding.load().lasad_decode_step_pages(a["q"], a["k"], a["v"], a["o"], _by(pages), a["io"], a["ot"], a["B"], a["Hq"], a["Hk"], a["d"], a["gh"],
                                                  a["gw"], a["pos"], a["rows"], a["wq"], a["wk"], a["shared"], a["eps"], a["rope"], a["pair"], a["base"],
                                                  a["window"], a["sinks"], a["scale"], a["ws"], a["bytes"], None)


POOLS = [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(table=None), dict(k=0x10008), dict(v=0x20004), dict(ks=0x30002), dict(vs=0x40001),
         dict(table=0x50002), dict(n=0), dict(n=-1), dict(pages=0), dict(pages=(1 << 24) + 1), dict(stride=-1), dict(v=0x10000), dict(vs=0x30000)]
SIZES = [dict(B=0), dict(B=-1), dict(Hk=0), dict(d=96), dict(d=256), dict(io=2), dict(ot=7), dict(io=0, ot=1), dict(Hq=1 << 16), dict(Hk=1 << 16),
         dict(rows=0x6002), dict(pos=-1), dict(pos=256), dict(B=(1 << 24) + 1)]
OPTIONS = [dict(gh=0), dict(gw=-1), dict(gh=1 << 16, gw=1 << 16), dict(rope=3), dict(pair=2), dict(base=1.0), dict(base=float("inf")), dict(eps=float("nan")),
           dict(eps=-1.0, wk=0x7000), dict(wk=0x7004), dict(pos=255, gw=8)]
MASKS = [dict(window=0), dict(sinks=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.0 ** 127.5), dict(Hq=3), dict(Hq=0)]
REFUSED = (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED)


def refused(status):
    assert status in REFUSED
    assert len(binding.load().lasad_last_error()) > 4


@pytest.mark.parametrize("call", [_append, _forward, _step])
@pytest.mark.parametrize("bad", POOLS, ids=lambda b: ",".join(b))
def test_pools_refused(call, bad):
    refused(call(pages=_struct(**bad)))


@pytest.mark.parametrize("call", [_append, _forward, _step])
def test_no_pool_refused(call):
    refused(call(pages=None))


@pytest.mark.parametrize("call", [_append, _forward, _step])
@pytest.mark.parametrize("bad", SIZES, ids=lambda b: ",".join(b))
def test_sizes_refused(call, bad):
    if "pos" in bad and bad["pos"] > 0 and call is _forward:
        bad = dict(pos=4 * 64)
    refused(call(**bad))


@pytest.mark.parametrize("call", [_append, _step])
@pytest.mark.parametrize("bad", OPTIONS, ids=lambda b: ",".join(b))
def test_options_refused(call, bad):
    refused(call(**bad))


@pytest.mark.parametrize("call", [_forward, _step])
@pytest.mark.parametrize("bad", MASKS, ids=lambda b: ",".join(b))
def test_masks_refused(call, bad):
    refused(call(**bad))


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(out=None), dict(q=0x1008), dict(k=0x2004), dict(v=0x3002), dict(out=0x4008), dict(lq=None), dict(lk=None), dict(lv=None),
    dict(lo=None), dict(lk=L(0, 126, 64)), dict(lv=L(0, -128, 64)), dict(lo=L(0, 0, 64)), dict(lo=L(0, 256, 32)), dict(n=-1), dict(starts=0x5002),
    dict(starts=None), dict(out=0x2000), dict(out=0x3000), dict(out=0x1000, ot=0), dict(out=0x1000, lo=L(0, 512, 64)), dict(q=None),
    dict(q=None, out=None, wq=0x7000), dict(n=(1 << 28) + 1)], ids=lambda b: ",".join(b))
def test_append_refused(bad):
    refused(_append(**bad))


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(o=None), dict(q=0x1008), dict(o=0x4008), dict(lq=None), dict(lo=None), dict(lo=L(0, 0, 64)), dict(lq=L(0, 254, 64)), dict(n=-1),
    dict(starts=0x5002), dict(starts=None), dict(o=0x1000), dict(n=(1 << 28) + 1), dict(ws=0x9004, bytes=1 << 30)], ids=lambda b: ",".join(b))
def test_forward_refused(bad):
    refused(_forward(**bad))


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=0x1008), dict(k=0x2008), dict(v=0x3008), dict(o=0x4004),
                                 dict(o=0x1000), dict(o=0x2000), dict(o=0x3000), dict(ws=0x9004, bytes=1 << 30)], ids=lambda b: ",".join(b))
def test_step_refused(bad):
    refused(_step(**bad))


def test_workspaces():
    lib = binding.load()
    size = lambda *a: lib.lasad_decode_step_pages_workspace_bytes(*a)
    assert size(1, 12, 12, 64, 5, 128, 1) == 0                              # few keys
    assert size(2, 16, 16, 64, 700, 16384, 64) > 0
    assert size(128, 20, 20, 64, 64, 4096, 0) == 0                          # enough workgroups
    assert lib.lasad_forward_pages_workspace_bytes(2, 16, 16, 64, 2, 1, 700, 16384, 64) == size(2, 16, 16, 64, 700, 16384, 64)
    for bad in ((0, 16, 16, 64, 700, 16384, 64), (2, 15, 16, 64, 700, 16384, 64), (2, 16, 16, 96, 700, 16384, 64), (2, 16, 16, 64, 0, 16384, 64),
                (2, 16, 16, 64, 700, 0, 64), (2, 16, 16, 64, 700, 16384, -1), (2, 16, 0, 64, 700, 16384, 64), ((1 << 24) + 1, 16, 16, 64, 700, 16384, 64)):
        assert size(*bad) == 0
    assert lib.lasad_forward_pages_workspace_bytes(2, 16, 16, 64, -1, 0, 700, 16384, 64) == 0
    assert lib.lasad_forward_pages_workspace_bytes(2, 16, 16, 64, 3, 1, 700, 16384, 64) == 0
    small = dict(pages=_struct(pages=700, stride=700), Hq=2, Hk=2, window=16384, ws=0x90000, bytes=16)
    assert _step(**small) == binding.ERR_WORKSPACE
    assert _forward(**small, starts=None, n=2, lq=L(0, 128, 64), lo=L(0, 128, 64)) == binding.ERR_WORKSPACE


def test_no_tokens_is_no_launch():
    assert _append(n=0, q=None, out=None, k=None, v=None) == binding.OK
    assert _forward(n=0, q=None, o=None) == binding.OK


def test_launches_beyond_a_grid():
    refused(_append(B=1 << 24, n=1, Hq=4096, Hk=2, lq=L(0, 1 << 18, 64), lo=L(0, 1 << 18, 64)))
    refused(_forward(B=1 << 24, n=1))


def test_binding_refuses():
    pages = binding.new_pages(4, 2, 64, device="cpu")
    table = torch.zeros(2, 3, dtype=torch.int32)
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    starts = torch.tensor([0, 2, 5], dtype=torch.int32)
    ok = dict(q=q, k=k, v=k, pages=pages, table=table, pos=0, grid_h=16, grid_w=16, row_starts=starts)
    p = pages
    for bad in (dict(v=k[:4]), dict(v=k.bfloat16()), dict(q=q.bfloat16()), dict(q=q[:4]), dict(table=table[:, ::2]), dict(table=table.long()),
                dict(table=table[0]), dict(row_starts=starts[:2]), dict(row_starts=starts.long()), dict(pos=torch.zeros(2)), dict(pos=starts),
                dict(pages=binding.new_pages(4, 3, 64, device="cpu")), dict(pages=(p.k.view(torch.uint8), *p[1:])), dict(pages=(p.v, p.k, *p[2:])),
                dict(pages=(*p[:2], p.k_scales.double(), p.v_scales)), dict(pages=(*p[:3], p.v_scales[:, :1])), dict(grid_h=1 << 40), dict(pos=1 << 40),
                dict(out=q[:4]), dict(q=None, out=q), dict(q=None, q_weight=torch.ones(64)), dict(k_weight=torch.ones(32)),
                dict(q_weight=torch.ones(64), k_weight=torch.ones(2, 64)), dict(q=q[0])):
        with pytest.raises((ValueError, TypeError)):
            binding.lasad_append_pages(**{**ok, **bad})
    ok = dict(q=q, pages=pages, table=table, pos=0, window=4, row_starts=starts)
    for bad in (dict(q=q[0]), dict(q=q.transpose(1, 2)), dict(table=table[:1].view(-1)), dict(window=1 << 31), dict(sinks=1 << 31), dict(out=q[:2]),
                dict(pages=binding.new_pages(4, 2, 32, device="cpu")), dict(row_starts=starts.float())):
        with pytest.raises(ValueError):
            binding.lasad_forward_pages(**{**ok, **bad})
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)
    ok = dict(q=q, k=k, v=k, pages=pages, table=table, pos=0, grid_h=16, grid_w=16, window=4)
    for bad in (dict(q=q[:1]), dict(q=q.transpose(0, 1)), dict(v=k[:1]), dict(k=k.bfloat16(), v=k.bfloat16()), dict(table=table[:1]), dict(window=1 << 32),
                dict(out=q[:1]), dict(pos=torch.zeros(3, dtype=torch.int32)), dict(k_weight=torch.ones(2, 64, dtype=torch.float64))):
        with pytest.raises(ValueError):
            binding.lasad_decode_step_pages(**{**ok, **bad})
    # right but for where they lie
    with pytest.raises(ValueError, match="GPU"):
        binding.lasad_decode_step_pages(**ok)


def test_the_order_of_a_page_of_values():
    """Position 16 b + 4 g + i lies at 16 g + 4 b + i."""
    assert sorted(pr.PLACE.tolist()) == list(range(64))
    for b in range(4):
        for g in range(4):
            for i in range(4):
                assert pr.PLACE[16 * b + 4 * g + i] == 16 * g + 4 * b + i


def test_the_reference_catches_mistakes():
    """A page that is not what an append leaves: a code a step off, a scale half of it, an earlier code that did not shrink."""
    gen = torch.Generator().manual_seed(1)
    y = torch.randn(10, 64, generator=gen, dtype=torch.float64)
    old = torch.zeros(64, 64, dtype=torch.float64)
    old[:20] = torch.randn(20, 64, generator=gen).mul(100).to(torch.float8_e4m3fn).double()
    scale0 = 2.0 ** -12                                    # too small for y: it grows
    power = 2.0 ** max(0, int(torch.log2(y.abs().max() / (448 * scale0)).ceil()))
    scale = scale0 * power
    new = old.clone()
    new[:20] = (old[:20].float() / power).to(torch.float8_e4m3fn).double()
    new[20:30] = (y / scale).to(torch.float8_e4m3fn).double()
    zero = torch.zeros_like(y)
    check = lambda codes, s: pr.check_stored(y, zero, old, scale0, codes, s, 20, "page")
    assert power >= 2
    check(new, scale)
    for bad, s in ((old.clone(), scale), (new, scale * 2), (new, scale / 2), (new, scale * 1.5)):
        with pytest.raises(AssertionError):
            check(bad, s)
    for i in range(3):
        bad = new.clone()
        bad[20 + i, i] = bad[20 + i, i] * 1.25
        with pytest.raises(AssertionError):
            check(bad, scale)
