"""The softmax layers' operators on tensors of more than 2^31 elements: addressing must be 64-bit.  Inputs are drawn on the GPU
from seeded generators; tokens at the start, on both sides of element offset 2^31 and at the end are compared with the 64-bit
reference, which is given the tokens that they depend on."""
import pytest
import torch

import softmax_layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
D, CUT = 64, 1 << 31


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


def normal(shape, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(shape, dtype=BF, device="cuda")
    for part in x.view(-1).split(1 << 28):
        part.normal_(generator=gen)
    return x


def check(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(want).all() and (err <= bound).all(), f"{what}: {float((err / bound).max()):.3g} of the bound"


def test_qk_forward_and_backward(lasad):
    B, n, Hq, W = 350, 4096, 24, 64
    q, k = normal((B, n, Hq, D), 1), normal((B, n, 1, D), 2)
    assert q.numel() > CUT
    w = [ref.draw((D,), F, i, 0.3) + 1 for i in (3, 4)]
    dev = [x.cuda() for x in w]
    yq, yk = lasad.lasad_forward_qk(q, k, W, W, *dev)
    gq, gk = normal(q.shape, 5), normal(k.shape, 6)
    dq, dk, _, _ = lasad.lasad_backward_qk(q, k, gq, gk, W, W, *dev, want_dweight=False)
    token = CUT // (Hq * D)
    for b, i0 in ((0, 0), (token // n, token % n - 20), (B - 1, n - 40)):
        at = (slice(b, b + 1), slice(i0, i0 + 40))
        pos = torch.arange(i0, i0 + 40)[None]
        for x, y, g, dx, wx, what in ((q, yq, gq, dq, w[0], "q"), (k, yk, gk, dk, w[1], "k")):
            x, g, wx = x[at].cpu().double(), g[at].cpu().double(), wx.double()
            want = ref.qk_row(x, wx, pos, W, 2, False, 10000.0, 1e-6)
            check(y[at], want, ref.qk_forward_bound(x, wx, 2, False, 1e-6, BF, want, n), f"{what} of {b}, {i0}")
            want = ref.qk_backward_reference(x, wx, g, pos, W, 2, False, 10000.0, 1e-6)[0]
            check(dx[at], want, ref.qk_backward_bound(x, wx, g, 2, False, 1e-6, BF, want, n)[0], f"d{what} of {b}, {i0}")


def test_window_forward_and_backward(lasad):
    n, H, w, s = 1450000, 24, 64, 2
    q, k, v, do = (normal((1, n, H, D), i) for i in (1, 2, 3, 4))
    assert q.numel() > CUT
    o, lse = lasad.lasad_forward_window(q, k, v, w, s, want_lse=True)
    dq, dk, dv = lasad.lasad_backward_window(q, k, v, o, lse, do, w, s)
    heads = [0, 11, H - 1]
    for t0 in (s, CUT // (H * D) - 20, n - 40):              # (the sinks' own gradients are sums over everything)
        queries = torch.arange(t0, min(n, t0 + 40 + w - 1))
        keys = torch.cat((torch.arange(s), torch.arange(max(s, t0 - w + 1), int(queries[-1]) + 1)))
        p, j = queries[:, None], keys[None]
        mask = ((j <= p) & ((p - j < w) | (j < s)))[None]
        x = [t[:, i][:, :, heads].cpu().double() for t, i in ((q, queries), (k, keys), (v, keys), (do, queries))]
        want, want_lse = ref.window_forward(*x[:3], mask, D ** -0.5)
        bound, lse_bound = ref.window_forward_bounds(*x[:3], mask, D ** -0.5, BF, BF, want, want_lse)
        check(o[:, queries][:, :, heads], want, bound, f"o from {t0}")
        check(lse[:, heads][:, :, queries], want_lse, lse_bound, f"lse from {t0}")
        grads = ref.window_backward(*x, mask, D ** -0.5)
        bounds = ref.window_backward_bounds(*x, mask, D ** -0.5, BF, BF, grads)
        first = int((keys == t0).nonzero()[0])
        check(dq[:, queries][:, :, heads], grads[0], bounds[0], f"dq from {t0}")
        for got, want, bound, what in ((dk, grads[1], bounds[1], "dk"), (dv, grads[2], bounds[2], "dv")):
            check(got[:, t0:t0 + 40][:, :, heads], want[:, first:first + 40], bound[:, first:first + 40], f"{what} from {t0}")


def test_window_step_over_a_long_cache(lasad):
    B, Hk, G, rows, s, scale = 2, 8, 2, 2200000, 4, 0.5
    w = rows - s
    kc, vc = normal((B, Hk, rows, D), 1), normal((B, Hk, rows, D), 2)
    assert kc.numel() > CUT
    q, k, v = normal((B, Hk * G, D), 3), normal((B, Hk, D), 4), normal((B, Hk, D), 5)
    pos = torch.tensor([5000001, 7654321], dtype=torch.int32)
    got = lasad.lasad_decode_step_window(q, k, v, kc, vc, pos.cuda(), w, s, scale=scale, out_dtype=F)
    cut = CUT // (rows * D)
    assert 0 < cut < B * Hk
    for bh in (0, cut - 1, cut, B * Hk - 1):
        b, h = bh // Hk, bh % Hk
        row = ref.cache_row(int(pos[b]), s, rows)
        assert torch.equal(kc[b, h, row], k[b, h]) and torch.equal(vc[b, h, row], v[b, h])
        K, V = kc[b, h].double(), vc[b, h].double()          # (every row is seen)
        for g in range(G):
            x = q[b, h * G + g].double()
            p = torch.softmax(K @ x * scale, 0)
            # as the reference's bound, with the additions that a lane makes: 32 splits of 4 wavefronts of 8 rows at a time, then joins
            top = float((K.abs() @ x.abs()).max()) * scale
            rel = 2 * (D + 8) * ref.U * (top + 1) + (4 * (rows // (32 * 32) + 100) + 16) * ref.U
            want = (p @ V).cpu()
            check(got[b, h * G + g], want, (p @ V.abs()).cpu() * rel + ref.stored(F, want), f"o of {bh}, {g}")
