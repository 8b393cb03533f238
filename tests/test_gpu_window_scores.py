"""The window attention where scores are not of unit variance, where inputs are views and where keys are not finite, in every kernel
of the forward and of the backward: few, middling and many queries, fp32 and bf16, all head dims."""
import math

import pytest
import torch

import softmax_layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
FAR = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


def check(got, want, bound, what):
    assert got.shape == want.shape and not got.isnan().any(), what
    err = (got.double() - want).abs()
    worst = float((err / bound.clamp(min=1e-300)).max())
    assert (err <= bound).all(), f"{what}: {worst:.3g} of the bound"


# dtype, d, batch rows, query heads, key heads; of 200 tokens: workgroups of 32 queries, of 64 (bf16), of 128
SIZES = [(BF, 64, 1, 2, 1), (BF, 64, 10, 16, 8), (BF, 64, 25, 16, 8), (BF, 32, 1, 3, 3), (BF, 32, 15, 16, 16), (BF, 32, 25, 16, 8),
         (BF, 128, 1, 2, 2), (BF, 128, 4, 16, 8), (F, 64, 1, 2, 1), (F, 64, 13, 16, 8), (F, 32, 13, 16, 16), (F, 128, 13, 16, 8)]
IDS = [f"{str(c[0])[6:]}-d{c[1]}-B{c[2]}-{c[3]}x{c[4]}" for c in SIZES]


def scored(size, kind, n=200, seed=3):
    """Inputs whose scores go as `kind` says; the scale; window and sinks."""
    dt, d, B, Hq, Hk = size
    q, k, v, do = (ref.draw((B, n, h, d), torch.float64, seed + i).cuda() for i, h in enumerate((Hq, Hk, Hk, Hq)))
    scale, window, sinks = d ** -0.5, FAR, 0
    j = torch.arange(n, dtype=torch.float64, device="cuda")
    if kind in ("rising", "falling", "rising in a window"):
        # a ramp along the keys through one channel: 7.7 in 32 keys (2^11); values shrink (grow) as much, so that every key has a part
        slope = -0.24 if kind == "falling" else 0.24
        q[..., 0] = 1.0
        k[..., 0] = (slope * j / scale)[None, :, None]
        v *= torch.exp(-slope * j)[None, :, None, None]
        if kind == "rising in a window":
            window, sinks = 70, 3
    elif kind == "steps":
        # flat but for one step of 6 (2^8.7) up every 64 keys
        q[..., 1] = 1.0
        k[..., 1] = (6.0 * torch.floor(j / 64) / scale)[None, :, None]
        v *= torch.exp(-6.0 * torch.floor(j / 64))[None, :, None, None]
    elif kind == "large scale":
        scale = 1.0                                       # (a standard deviation of sqrt(d))
    else:
        assert kind == "small scale"
        scale = 1e-3
    return [t.to(dt) for t in (q, k, v, do)], scale, window, sinks


@pytest.mark.parametrize("kind", ["rising", "falling", "rising in a window", "steps", "large scale", "small scale"])
@pytest.mark.parametrize("size", SIZES, ids=IDS)
def test_scores_that_move_the_maximum(lasad, size, kind):
    (q, k, v, do), scale, window, sinks = scored(size, kind)
    B, n = q.shape[:2]
    given = None if scale == size[1] ** -0.5 else scale
    kw = dict(window=window, sinks=sinks, scale=given)
    o, lse = lasad.lasad_forward_window(q, k, v, out_dtype=F, want_lse=True, **kw)
    stored = lasad.lasad_forward_window(q, k, v, **kw)
    got = lasad.lasad_backward_window(q, k, v, stored, lse, do, grad_dtype=F, **kw)
    mask = ref.seen_mask(n, n, 0, window, sinks, None, B).cuda()
    x = [t.double() for t in (q, k, v, do)]
    if kind in ("rising", "steps"):                       # the last query's maximum does rise by more than 2^8 from block to block
        s = (x[0][0, -1, 0] @ x[1][0, :, 0].T) * scale / math.log(2)
        tops = s[:192].view(-1, 64).amax(-1).cummax(0).values
        assert (tops[1:] - tops[:-1] > 8.0).any() if kind == "steps" else (tops[1:] - tops[:-1] > 8.0).all()
    want, want_lse = ref.window_forward(*x[:3], mask, scale)
    bound, lse_bound = ref.window_forward_bounds(*x[:3], mask, scale, size[0], F, want, want_lse)
    check(o, want, bound, "o")
    check(lse, want_lse, lse_bound, "lse")
    grads = ref.window_backward(*x, mask, scale)
    for g, w, b, what in zip(got, grads, ref.window_backward_bounds(*x, mask, scale, size[0], F, grads), ("dq", "dk", "dv")):
        check(g, w, b, what)


@pytest.mark.parametrize("size", SIZES, ids=IDS)
def test_views_and_broadcast_inputs(lasad, size):
    """q, k, v as a projection's views, heads-first outputs and gradients, keys of one row for all, one gradient for all tokens: the
    numbers of dense tensors, bit for bit."""
    dt, d, B, Hq, Hk = size
    n, w, s = 183, 50, 3
    proj = ref.draw((B, n, Hq + 2 * Hk, d), dt, 3).cuda()
    q, k, v = proj.split((Hq, Hk, Hk), 2)
    do = ref.draw((B, Hq, n, d), dt, 4).cuda().transpose(1, 2)
    dense = [t.contiguous() for t in (q, k, v)]
    want, lse = lasad.lasad_forward_window(*dense, w, s, want_lse=True)
    out = torch.full((B, Hq, n, d), float("nan"), dtype=dt, device="cuda").transpose(1, 2)
    got, lse2 = lasad.lasad_forward_window(q, k, v, w, s, out=out, want_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    dwant = lasad.lasad_backward_window(*dense, want, lse, do.contiguous(), w, s)
    grad = torch.full_like(proj, float("nan"))
    dgot = lasad.lasad_backward_window(q, k, v, got, lse, do, w, s, grads=grad.split((Hq, Hk, Hk), 2))
    assert all(torch.equal(a, b) for a, b in zip(dgot, dwant)) and not grad.isnan().any()
    kb, vb, gb = k[:1].expand(B, n, Hk, d), v[:1].expand(B, n, Hk, d), do[:, :1].expand(B, n, Hq, d)
    o1, l1 = lasad.lasad_forward_window(q, kb, vb, w, s, want_lse=True)
    o2, l2 = lasad.lasad_forward_window(q, kb.contiguous(), vb.contiguous(), w, s, want_lse=True)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    a = lasad.lasad_backward_window(q, kb, vb, o1, l1, gb, w, s)
    b = lasad.lasad_backward_window(q, kb.contiguous(), vb.contiguous(), o1, l1, gb.contiguous(), w, s)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("size", SIZES, ids=IDS)
def test_rows_that_see_a_key_that_is_not_finite(lasad, size, value):
    """k_j[7] = value: a score of +infinity or NaN makes the row NaN, one of -infinity takes the key out of it; dq_i[7] has the term
    dS_ij k_j[7], which is not finite either way.  v_j[7] = value: o_i[7] is not finite, and all of dq_i with it (through dP and delta)."""
    dt, d, B, Hq, Hk = size
    n, w, s = 200, 90, 2
    q, k, v, do = (ref.draw((B, n, h, d), dt, 3 + i).cuda() for i, h in enumerate((Hq, Hk, Hk, Hq)))
    G = Hq // Hk
    mask = ref.seen_mask(n, n, 0, w, s)[0].cuda()
    for j in (1, 100):
        sees = mask[:, j]
        bad = k.clone()
        bad[0, j, 0, 7] = value
        o, lse = lasad.lasad_forward_window(q, bad, v, w, s, want_lse=True)
        dq = lasad.lasad_backward_window(q, bad, v, o, lse, do, w, s)[0]
        rows, scores = o[0, sees, :G], q[0, sees, :G, 7].float() * value
        lost = ~(scores < 0)
        assert rows[lost].isnan().all() and rows[~lost].isfinite().all()      # (every row sees another key too)
        assert lse[0, :G].T[sees][lost].isnan().all() and lse[0, :G].T[sees][~lost].isfinite().all()
        assert not dq[0, sees, :G, 7].isfinite().any()
        assert dq[0, ~sees].isfinite().all() and o[0, ~sees].isfinite().all() and dq[0, :, G:].isfinite().all() and dq[1:].isfinite().all()
        bad = v.clone()
        bad[0, j, 0, 7] = value
        o, lse = lasad.lasad_forward_window(q, k, bad, w, s, want_lse=True)
        dq = lasad.lasad_backward_window(q, k, bad, o, lse, do, w, s)[0]
        assert not o[0, sees, :G, 7].isfinite().any() and o[0, sees, :G, :7].isfinite().all() and o[0, sees, :G, 8:].isfinite().all()
        assert not dq[0, sees, :G].isfinite().any() and dq[0, ~sees].isfinite().all() and dq[1:].isfinite().all() and lse.isfinite().all()


@pytest.mark.parametrize("kind,n", [("rising", 200), ("falling", 200), ("steps", 200), ("large scale", 200), ("small scale", 200), ("large scale", 2300)])
@pytest.mark.parametrize("size", [(BF, 64, 2, 2, 1), (BF, 32, 1, 3, 3), (BF, 128, 2, 8, 2), (F, 64, 1, 5, 1), (F, 128, 30, 16, 8)],
                         ids=lambda c: f"{str(c[0])[6:]}-d{c[1]}-B{c[2]}-{c[3]}x{c[4]}")
def test_steps(lasad, size, kind, n):
    (q, k, v, _), scale, window, sinks = scored(size, kind, n)
    given = None if scale == size[1] ** -0.5 else scale
    caches = [x.transpose(1, 2).clone(memory_format=torch.contiguous_format) for x in (k, v)]
    last = [x[:, -1].contiguous() for x in (q, k, v)]
    got = lasad.lasad_decode_step_window(*last, *caches, n - 1, window, sinks, scale=given, out_dtype=F)
    x = [t.double() for t in (q[:, -1:], k, v)]
    mask = torch.ones(size[2], 1, n, dtype=torch.bool, device="cuda")
    want, want_lse = ref.window_forward(*x, mask, scale)
    check(got[:, None], want, ref.window_forward_bounds(*x, mask, scale, F, F, want, want_lse)[0], "o")     # (no rounded operand)
