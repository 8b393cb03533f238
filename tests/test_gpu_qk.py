"""Head norms with raster rotation on the GPU against the 64-bit reference: types, layouts, positions, weights, gradients."""
import pytest
import torch

import softmax_layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
BASE, EPS = 10000.0, 1e-6


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


def weights(kind, Hq, Hk, d):
    if kind == "none":
        return None, None
    shapes = ((d,), (d,)) if kind == "shared" else ((Hq, d), (Hk, d))
    return tuple(ref.draw(s, F, 71 + i, 0.3) + 1 for i, s in enumerate(shapes))


def heads_of(w, x):
    return None if w is None else w.double()


# dtype, out dtype, d, Hq, Hk, B, H, W, start, n, rope, halves, weights, eps
CASES = [
    (BF, BF, 64, 12, 12, 2, 16, 16, 0, 256, 2, False, "shared", EPS),
    (BF, BF, 64, 16, 4, 3, 24, 23, 101, 311, 2, True, "heads", EPS),
    (BF, F, 64, 5, 5, 1, 9, 7, 0, 63, 1, True, "heads", EPS),
    (F, F, 64, 20, 4, 2, 24, 23, 13, 77, 1, False, "shared", EPS),
    (F, F, 64, 3, 1, 5, 1, 19, 18, 1, 2, True, "none", EPS),
    (BF, BF, 32, 6, 2, 4, 5, 31, 7, 40, 2, True, "shared", EPS),
    (F, F, 32, 33, 33, 2, 5, 31, 7, 17, 1, True, "heads", EPS),
    (BF, BF, 128, 7, 1, 2, 40, 3, 5, 29, 2, False, "heads", EPS),
    (F, F, 128, 24, 8, 1, 64, 64, 4000, 96, 2, True, "none", EPS),
    (BF, BF, 64, 12, 12, 1, 16, 16, 0, 100, 0, False, "heads", EPS),
    (BF, BF, 64, 12, 4, 2, 16, 16, 3, 50, 2, False, "none", -1.0),
    (F, F, 64, 1, 1, 1, 1, 1, 0, 1, 2, False, "shared", 1e-2),
    (BF, BF, 64, 16, 16, 16, 24, 24, 0, 576, 2, False, "shared", EPS),      # more tokens than one a workgroup
    (F, F, 64, 4, 2, 1, 1 << 15, 1 << 15, (1 << 30) - 40, 40, 1, False, "shared", EPS),     # far positions
]
IDS = [f"{str(c[0])[6:]}-{str(c[1])[6:]}-d{c[2]}-{c[3]}x{c[4]}-B{c[5]}-n{c[9]}-rope{c[10]}{'h' if c[11] else 'a'}-{c[12]}" for c in CASES]


def inputs(c, seed=5):
    dt, _, d, Hq, Hk, B, H, W, start, n = c[:10]
    q, k = ref.draw((B, n, Hq, d), dt, seed), ref.draw((B, n, Hk, d), dt, seed + 1)
    pos = (start + torch.arange(n))[None].expand(B, n)
    return q, k, pos, weights(c[12], Hq, Hk, d)


def check(got, want, bound, what):
    got = got.double().cpu()
    err = (got - want).abs()
    worst = (err / bound.clamp(min=1e-300)).max() if got.numel() else 0.0
    assert torch.isfinite(got).all() and (err <= bound).all(), f"{what}: {float(worst):.3g} of the bound"


def kwargs(c, ws):
    return dict(q_weight=None if ws[0] is None else ws[0].cuda(), k_weight=None if ws[1] is None else ws[1].cuda(),
                norm_eps=c[13], rope=c[10], pairing=int(c[11]), rope_base=BASE)


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_forward(lasad, c):
    q, k, pos, ws = inputs(c)
    got = lasad.lasad_forward_qk(q.cuda(), k.cuda(), c[6], c[7], start_pos=c[8], out_dtype=c[1], **kwargs(c, ws))
    for x, w, y, what in zip((q, k), ws, got, "qk"):
        x, w = x.double(), heads_of(w, x)
        want = ref.qk_row(x, w, pos, c[7], c[10], c[11], BASE, c[13])
        assert y.dtype == c[1]
        check(y, want, ref.qk_forward_bound(x, w, c[10], c[11], c[13], c[1], want, c[8] + c[9]), what)


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_backward(lasad, c):
    q, k, pos, ws = inputs(c)
    gs = ref.draw(q.shape, q.dtype, 31), ref.draw(k.shape, k.dtype, 32)
    got = lasad.lasad_backward_qk(q.cuda(), k.cuda(), gs[0].cuda(), gs[1].cuda(), c[6], c[7], start_pos=c[8], grad_dtype=c[1],
                                  **kwargs(c, ws))
    for i, (x, w, g, what) in enumerate(zip((q, k), ws, gs, "qk")):
        x, g, w = x.double(), g.double(), heads_of(w, x)
        at_ones = w if w is not None else torch.ones(x.shape[2:], dtype=torch.float64)       # (no weight: the gradient at ones)
        dx, dw = ref.qk_backward_reference(x, at_ones, g, pos, c[7], c[10], c[11], BASE, c[13])
        bound, term = ref.qk_backward_bound(x, w, g, c[10], c[11], c[13], c[1], dx, c[8] + c[9])
        check(got[i], dx, bound, "d" + what)
        if c[13] < 0:
            assert got[2 + i] is None
            continue
        axes = tuple(range(4 - at_ones.dim()))
        # (added up in runs of at most 8 tokens and 32 heads a lane, 4 wavefronts, then in runs of at most 36 and 16 lanes)
        adds = (8 + 32 + 4 + 36 + 16) * ref.U * (ref.pair_size(g, c[10], c[11]) * (x / torch.sqrt((x * x).mean(-1, keepdim=True) + c[13])).abs())
        assert got[2 + i].shape == at_ones.shape
        check(got[2 + i], dw, (term + adds).sum(axes), "dw" + what)


def test_weight_gradients_can_be_left_out(lasad):
    c = CASES[1]
    q, k, pos, ws = inputs(c)
    gs = ref.draw(q.shape, q.dtype, 31).cuda(), ref.draw(k.shape, k.dtype, 32).cuda()
    a = lasad.lasad_backward_qk(q.cuda(), k.cuda(), *gs, c[6], c[7], start_pos=c[8], **kwargs(c, ws))
    b = lasad.lasad_backward_qk(q.cuda(), k.cuda(), *gs, c[6], c[7], start_pos=c[8], want_dweight=False, **kwargs(c, ws))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and b[2] is None and b[3] is None


@pytest.mark.parametrize("dtype", [BF, F])
def test_views_of_a_projection_heads_first_and_broadcast_inputs(lasad, dtype):
    B, n, Hq, Hk, d, H, W = 2, 37, 6, 2, 64, 8, 9
    kw = dict(q_weight=weights("heads", Hq, Hk, d)[0].cuda(), k_weight=weights("heads", Hq, Hk, d)[1].cuda(), start_pos=5)
    proj = ref.draw((B, n, Hq + 2 * Hk, d), dtype, 3).cuda()
    q, k = proj[:, :, :Hq], proj[:, :, Hq:Hq + Hk]
    want = lasad.lasad_forward_qk(q.contiguous(), k.contiguous(), H, W, **kw)
    g = tuple(ref.draw(t.shape, dtype, 8).cuda() for t in (q, k))
    dwant = lasad.lasad_backward_qk(q.contiguous(), k.contiguous(), *g, H, W, **kw)
    # views in, heads-first tensors out
    outs = tuple(torch.full((B, t.shape[2], n, d), float("nan"), dtype=dtype, device="cuda").transpose(1, 2) for t in (q, k))
    got = lasad.lasad_forward_qk(q, k, H, W, out=outs, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    hf = tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in g)
    dgot = lasad.lasad_backward_qk(q, k, *hf, H, W, grads=tuple(torch.empty_like(o) for o in outs), **kw)
    assert all(torch.equal(a, b) for a, b in zip(dgot, dwant))
    # one row for all batches, one gradient for all tokens (stride 0)
    one = q[:1].expand(B, n, Hq, d)
    ga = g[0][:, :1].expand(B, n, Hq, d)
    a = lasad.lasad_forward_qk(one, k, H, W, **kw)
    b = lasad.lasad_forward_qk(one.contiguous(), k, H, W, **kw)
    assert torch.equal(a[0], b[0])
    a = lasad.lasad_backward_qk(one, k, ga, g[1], H, W, **kw)
    b = lasad.lasad_backward_qk(one.contiguous(), k, ga.contiguous(), g[1], H, W, **kw)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    # in place, inside the projection
    before = proj.clone()
    lasad.lasad_forward_qk(q, k, H, W, out=(q, k), **kw)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(proj[:, :, Hq + Hk:], before[:, :, Hq + Hk:])


@pytest.mark.parametrize("dtype,d,halves", [(BF, 64, False), (BF, 128, True), (F, 32, True), (F, 64, False)])
def test_single_tokens(lasad, dtype, d, halves):
    B, Hq, Hk, H, W = 37, 6, 3, 11, 13
    q, k = ref.draw((B, Hq, d), dtype, 1).cuda(), ref.draw((B, Hk, d), dtype, 2).cuda()
    kw = dict(q_weight=weights("shared", Hq, Hk, d)[0].cuda(), k_weight=weights("shared", Hq, Hk, d)[1].cuda(), pairing=int(halves))
    # one position for all: the forward's row, bit for bit
    a = lasad.lasad_decode_step_qk(q, k, H, W, 77, **kw)
    b = lasad.lasad_forward_qk(q[:, None], k[:, None], H, W, start_pos=77, **kw)
    assert all(torch.equal(x, y[:, 0]) for x, y in zip(a, b))
    # a position for each row; rows off the grid stay as they were
    pos = (torch.arange(B, dtype=torch.int32) * 31) % (H * W)
    pos[3], pos[9], pos[20] = -1, H * W, -2 ** 31
    out = tuple(torch.full_like(t, 7.0) for t in (q, k))
    got = lasad.lasad_decode_step_qk(q, k, H, W, pos.cuda(), out=out, **kw)
    for r in range(B):
        p = int(pos[r])
        if not 0 <= p < H * W:
            assert all((t[r] == 7.0).all() for t in got)
            continue
        want = lasad.lasad_decode_step_qk(q[r:r + 1], k[r:r + 1], H, W, p, **kw)
        assert all(torch.equal(x[r], y[0]) for x, y in zip(got, want))
    # in place
    want = lasad.lasad_decode_step_qk(q, k, H, W, 5, **kw)
    lasad.lasad_decode_step_qk(q, k, H, W, 5, out=(q, k), **kw)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rows_of_zeros_infinity_and_nan_stay_with_their_row(lasad):
    q, k = ref.draw((1, 8, 4, 64), BF, 1), ref.draw((1, 8, 4, 64), BF, 2)
    clean = lasad.lasad_forward_qk(q.cuda(), k.cuda(), 2, 4)[0]
    q[0, 2, 1] = 0.0
    q[0, 3, 2, 5] = float("inf")
    q[0, 4, 0, 7] = float("nan")
    got = lasad.lasad_forward_qk(q.cuda(), k.cuda(), 2, 4)[0]
    assert (got[0, 2, 1] == 0).all() and got[0, 4, 0].isnan().all()
    same = torch.ones(8, 4, dtype=torch.bool)
    same[2, 1] = same[3, 2] = same[4, 0] = False
    assert torch.equal(got[0].cpu()[same], clean[0].cpu()[same])


def test_no_tokens(lasad):
    e = torch.empty(2, 0, 4, 64, device="cuda", dtype=BF)
    w = torch.ones(4, 64, device="cuda")
    assert lasad.lasad_forward_qk(e, e, 3, 3)[0].shape == e.shape
    g = lasad.lasad_backward_qk(e, e, e, e, 3, 3, q_weight=w, k_weight=w)
    assert g[0].shape == e.shape and (g[2] == 0).all() and (g[3] == 0).all()


def test_another_stream_and_graph_replays(lasad):
    c = CASES[1]
    q, k, pos, ws = inputs(c)
    kw = kwargs(c, ws)
    H, W, start = c[6], c[7], c[8]
    q, k = q.cuda(), k.cuda()
    g = tuple(ref.draw(t.shape, BF, 4).cuda() for t in (q, k))
    want = lasad.lasad_forward_qk(q, k, H, W, start_pos=start, **kw)
    dwant = lasad.lasad_backward_qk(q, k, *g, H, W, start_pos=start, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lasad.lasad_forward_qk(q, k, H, W, start_pos=start, stream=side, **kw)
    dgot = lasad.lasad_backward_qk(q, k, *g, H, W, start_pos=start, stream=side, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *dgot), (*want, *dwant)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = lasad.lasad_forward_qk(q, k, H, W, start_pos=start, **kw)
        dgot = lasad.lasad_backward_qk(q, k, *g, H, W, start_pos=start, **kw)
    for i in range(3):
        q.copy_(ref.draw(q.shape, BF, 90 + i))
        want = lasad.lasad_forward_qk(q, k, H, W, start_pos=start, **kw)
        dwant = lasad.lasad_backward_qk(q, k, *g, H, W, start_pos=start, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, *dgot), (*want, *dwant)))
