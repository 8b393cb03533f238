"""Attention with a window and sinks on the GPU against the 64-bit reference: types, head layouts, lengths from nothing to
several tiles, masks that leave rows empty, layouts, gradients, single tokens against a cache that goes round."""
import pytest
import torch

import softmax_layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


# dtype, out dtype, d, Hq, Hk, B, start, n, m, window, sinks, lens
CASES = [
    (BF, BF, 64, 2, 2, 1, 0, 256, 256, 128, 1, None),
    (BF, F, 64, 6, 2, 2, 101, 147, 248, 96, 16, None),
    (BF, BF, 64, 4, 1, 3, 0, 300, 300, 33, 0, [300, 0, 77]),             # a row without keys; queries past the keys
    (F, F, 64, 4, 2, 2, 37, 131, 168, 50, 3, [168, 20]),
    (F, F, 64, 1, 1, 1, 0, 1, 1, 1, 0, None),
    (BF, BF, 64, 3, 3, 2, 500, 1, 501, 64, 4, None),                     # one query
    (BF, BF, 64, 2, 1, 1, 0, 200, 200, 1, 0, None),                      # every query sees itself
    (BF, BF, 64, 2, 1, 1, 0, 200, 200, 1, 70, None),                     # and more sinks than a tile has keys
    (BF, BF, 64, 2, 2, 1, 0, 190, 190, 2 ** 31 - 1, 0, None),            # all keys up to the query's
    (BF, BF, 64, 2, 2, 1, 0, 190, 190, 40, 2 ** 31 - 1, None),           # (all are sinks)
    (BF, BF, 64, 2, 1, 2, 64, 65, 400, 63, 5, None),                     # keys beyond the last query
    (BF, BF, 64, 2, 1, 1, 400, 70, 130, 90, 0, None),                    # keys that end long before the queries: nothing seen
    (BF, BF, 64, 2, 1, 1, 400, 70, 130, 90, 9, None),                    # but the sinks
    (BF, BF, 32, 4, 4, 1, 3, 129, 132, 65, 2, None),
    (F, F, 32, 5, 1, 1, 0, 100, 100, 31, 1, None),
    (BF, F, 128, 4, 2, 1, 10, 140, 150, 77, 1, [143]),
    (F, F, 128, 2, 1, 2, 0, 97, 97, 40, 4, None),
    (BF, BF, 64, 6, 2, 1, 0, 1100, 1100, 100, 4, None),                  # the sinks' queries in parts
    (F, F, 64, 2, 1, 1, 0, 700, 700, 64, 130, None),                     # two tiles of sinks, in parts
]
# The same masks with heads enough for workgroups of 128 queries and keys (the ones above have 32): (case, batch rows, heads, key heads)
MANY = [(CASES[i], B, Hq, Hk) for i, B, Hq, Hk in ((0, 12, 16, 16), (1, 16, 12, 12), (2, 9, 32, 16), (3, 13, 16, 16), (6, 8, 32, 16), (7, 8, 32, 32),
                                                   (8, 16, 16, 8), (9, 8, 32, 16), (10, 16, 16, 16), (11, 32, 16, 8), (12, 32, 16, 16), (13, 10, 16, 16),
                                                   (14, 16, 32, 16), (15, 13, 16, 8), (16, 16, 32, 16), (17, 4, 12, 4), (18, 4, 24, 24))]
# and enough for the forward's workgroups of 128 in bf16 (those above have 64)
MANY += [(CASES[i], B, Hq, Hk) for i, B, Hq, Hk in ((0, 25, 16, 16), (1, 34, 12, 12), (2, 17, 16, 8), (4, 100, 16, 16), (5, 50, 16, 8), (6, 13, 32, 16), (7, 13, 32, 32),
                                                   (8, 25, 16, 8), (9, 25, 16, 16), (10, 50, 16, 16), (11, 50, 16, 8), (12, 50, 16, 16), (13, 13, 32, 16),
                                                   (17, 8, 12, 4))]
IDS = [f"{str(c[0])[6:]}-{str(c[1])[6:]}-d{c[2]}-{c[3]}x{c[4]}-B{c[5]}-{c[6]}+{c[7]}of{c[8]}-w{c[9]}-s{c[10]}{'-lens' if c[11] else ''}" for c in CASES]


def inputs(c, seed=7):
    dt, _, d, Hq, Hk, B, start, n, m = c[:9]
    q = ref.draw((B, n, Hq, d), dt, seed)
    k, v = ref.draw((B, m, Hk, d), dt, seed + 1), ref.draw((B, m, Hk, d), dt, seed + 2)
    return q, k, v, ref.seen_mask(n, m, start, c[9], c[10], c[11], B)


def check(got, want, bound, what):
    got = got.double().cpu()
    empty = want == -float("inf")
    assert torch.equal(got == -float("inf"), empty), what
    err = torch.where(empty, 0.0, (got - want).abs())
    assert got.shape == want.shape and not got.isnan().any(), what
    worst = float((err / bound.clamp(min=1e-300)).max()) if got.numel() else 0.0
    assert (err <= bound).all(), f"{what}: {worst:.3g} of the bound"


def lens_of(c):
    return None if c[11] is None else torch.tensor(c[11], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_forward(lasad, c):
    q, k, v, mask = inputs(c)
    o, lse = lasad.lasad_forward_window(q.cuda(), k.cuda(), v.cuda(), c[9], c[10], start_pos=c[6], kv_lens=lens_of(c), out_dtype=c[1], want_lse=True)
    x = [t.double() for t in (q, k, v)]
    want, want_lse = ref.window_forward(*x, mask, c[2] ** -0.5)
    bound, lse_bound = ref.window_forward_bounds(*x, mask, c[2] ** -0.5, c[0], c[1], want, want_lse)
    assert o.dtype == c[1]
    check(o, want, bound, "o")
    check(lse, want_lse, lse_bound, "lse")
    none = ~mask.any(-1)
    assert (o.cpu()[none] == 0).all()


@pytest.mark.parametrize("many", MANY, ids=lambda m: f"{str(m[0][0])[6:]}-d{m[0][2]}-{m[2]}x{m[3]}-B{m[1]}-{m[0][6]}+{m[0][7]}of{m[0][8]}-w{m[0][9]}-s{m[0][10]}")
def test_many_heads(lasad, many):
    """Forward and backward, with the reference's 64-bit arithmetic on the GPU."""
    c, B, Hq, Hk = many
    lens = None if c[11] is None else (c[11] * B)[:B]
    c = (*c[:3], Hq, Hk, B, *c[6:11], lens)
    q, k, v, mask = inputs(c)
    do = ref.draw(q.shape, q.dtype, 55)
    dev, mask = [t.cuda() for t in (q, k, v, do)], mask.cuda()
    kw = dict(start_pos=c[6], kv_lens=lens_of(c))
    o, lse = lasad.lasad_forward_window(*dev[:3], c[9], c[10], want_lse=True, **kw)
    o32 = lasad.lasad_forward_window(*dev[:3], c[9], c[10], out_dtype=F, **kw)
    got = lasad.lasad_backward_window(*dev[:3], o, lse, dev[3], c[9], c[10], grad_dtype=c[1], **kw)
    x = [t.double() for t in dev]
    want, want_lse = ref.window_forward(*x[:3], mask, c[2] ** -0.5)
    bound, lse_bound = ref.window_forward_bounds(*x[:3], mask, c[2] ** -0.5, c[0], F, want, want_lse)
    check(o32, want.cpu(), bound.cpu(), "o")
    check(lse, want_lse.cpu(), lse_bound.cpu(), "lse")
    assert torch.equal(o, o32.to(c[0]))
    grads = ref.window_backward(*x, mask, c[2] ** -0.5)
    for g, w, b, what in zip(got, grads, ref.window_backward_bounds(*x, mask, c[2] ** -0.5, c[0], c[1], grads), ("dq", "dk", "dv")):
        check(g, w.cpu(), b.cpu(), what)


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_backward(lasad, c):
    q, k, v, mask = inputs(c)
    do = ref.draw(q.shape, q.dtype, 55)
    dev = [t.cuda() for t in (q, k, v)]
    kw = dict(start_pos=c[6], kv_lens=lens_of(c))
    o, lse = lasad.lasad_forward_window(*dev, c[9], c[10], want_lse=True, **kw)
    got = lasad.lasad_backward_window(*dev, o, lse, do.cuda(), c[9], c[10], grad_dtype=c[1], **kw)
    x = [t.double() for t in (q, k, v)]
    want = ref.window_backward(*x, do.double(), mask, c[2] ** -0.5)
    bounds = ref.window_backward_bounds(*x, do.double(), mask, c[2] ** -0.5, c[0], c[1], want)
    for g, w, b, what in zip(got, want, bounds, ("dq", "dk", "dv")):
        assert g.dtype == c[1]
        check(g, w, b, what)
    unseen = ~mask.any(1)
    assert (got[1].cpu()[unseen] == 0).all() and (got[2].cpu()[unseen] == 0).all()


def test_results_are_the_same_again(lasad):
    c = CASES[17]
    dev = [t.cuda() for t in inputs(c)[:3]]
    do = ref.draw(dev[0].shape, BF, 5).cuda()

    def once():
        o, lse = lasad.lasad_forward_window(*dev, c[9], c[10], want_lse=True)
        return (o, lse, *lasad.lasad_backward_window(*dev, o, lse, do, c[9], c[10]))
    assert all(torch.equal(a, b) for a, b in zip(once(), once()))


@pytest.mark.parametrize("dtype", [BF, F])
def test_views_heads_first_and_broadcast_inputs(lasad, dtype):
    B, n, Hq, Hk, d, w, s = 2, 83, 6, 2, 64, 40, 3
    proj = ref.draw((B, n, Hq + 2 * Hk, d), dtype, 3).cuda()
    q, k, v = proj[:, :, :Hq], proj[:, :, Hq:Hq + Hk], proj[:, :, Hq + Hk:]
    do = ref.draw((B, Hq, n, d), dtype, 4).cuda().transpose(1, 2)
    dense = [t.contiguous() for t in (q, k, v)]
    want, lse = lasad.lasad_forward_window(*dense, w, s, want_lse=True)
    out = torch.empty((B, Hq, n, d), dtype=dtype, device="cuda").transpose(1, 2)
    got, lse2 = lasad.lasad_forward_window(q, k, v, w, s, out=out, want_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    dwant = lasad.lasad_backward_window(*dense, want, lse, do.contiguous(), w, s)
    grad = torch.empty_like(proj)
    dgot = lasad.lasad_backward_window(q, k, v, got, lse, do, w, s, grads=(grad[:, :, :Hq], grad[:, :, Hq:Hq + Hk], grad[:, :, Hq + Hk:]))
    assert all(torch.equal(a, b) for a, b in zip(dgot, dwant))
    # one set of keys for all batch rows, one gradient for all queries (stride 0)
    kb, vb, gb = k[:1].expand(B, n, Hk, d), v[:1].expand(B, n, Hk, d), do[:, :1].expand(B, n, Hq, d)
    o1, l1 = lasad.lasad_forward_window(q, kb, vb, w, s, want_lse=True)
    o2, l2 = lasad.lasad_forward_window(q, kb.contiguous(), vb.contiguous(), w, s, want_lse=True)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    a = lasad.lasad_backward_window(q, kb, vb, o1, l1, gb, w, s)
    b = lasad.lasad_backward_window(q, kb.contiguous(), vb.contiguous(), o1, l1, gb.contiguous(), w, s)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B", [2, 160, 200])
def test_what_is_not_seen_has_no_part(lasad, dtype, value, B):
    """Keys past a row's length, past the last query and before all windows hold `value`: nothing changes.  One key in the middle
    does: only its own queries change."""
    n, m, start, w, s, d = 150, 400, 130, 40, 2, 64
    q, k, v = ref.draw((B, n, 2, d), dtype, 1), ref.draw((B, m, 1, d), dtype, 2), ref.draw((B, m, 1, d), dtype, 3)
    do = ref.draw(q.shape, dtype, 4)
    lens = [400, 200] + [400] * (B - 2)
    mask = ref.seen_mask(n, m, start, w, s, lens, B)
    kw = dict(start_pos=start, kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))

    def run(q, k, v, do):
        dev = [t.cuda() for t in (q, k, v)]
        o, lse = lasad.lasad_forward_window(*dev, w, s, want_lse=True, **kw)
        return [t.cpu() for t in (o, lse, *lasad.lasad_backward_window(*dev, o, lse, do.cuda(), w, s, **kw))]
    clean = run(q, k, v, do)
    k1, v1 = k.clone(), v.clone()
    hidden = ~mask.any(1)
    k1[hidden], v1[hidden] = value, value
    assert hidden.any() and all(torch.equal(a, b) for a, b in zip(run(q, k1, v1, do), clean))
    for j, in_k in ((185, False), (185, True), (1, False)):
        k1, v1 = k.clone(), v.clone()
        (k1 if in_k else v1)[0, j, 0, 7] = value
        got = run(q, k1, v1, do)
        blind = ~mask[0, :, j]
        assert blind.any() == (j >= s) and mask[0, :, j].any()           # (a sink is seen by all)
        for a, b in zip((got[0][0], got[2][0]), (clean[0][0], clean[2][0])):
            assert torch.equal(a[blind], b[blind])
        seen = got[0][0][~blind]
        assert not seen.isfinite().all(-1).any() if not in_k else True
        if not in_k:
            assert (~seen[..., 7].isfinite()).all() and seen[..., 8].isfinite().all()      # its channel and no other
        assert all(torch.equal(a[1], b[1]) for a, b in zip(got, clean))
    # a query, or its gradient, that is not finite: only the keys that it sees change
    for x in (0, 3):
        ins = [t.clone() for t in (q, k, v, do)]
        ins[x][0, 60, 1, 9] = value
        got = run(*ins)
        blind = ~mask[0, 60]
        assert blind.any() and all(torch.equal(got[i][0][blind], clean[i][0][blind]) for i in (3, 4))
        assert not got[3][0][~blind].isfinite().all(-1).any()
        if x == 3:
            assert not got[4][0][~blind][..., 9].isfinite().any()
        others = torch.arange(n) != 60
        assert torch.equal(got[2][0][others], clean[2][0][others]) and torch.equal(got[0][0][others], clean[0][0][others])


def test_nothing_at_all(lasad):
    q, k = torch.empty(2, 0, 4, 64, device="cuda", dtype=BF), torch.ones(2, 9, 2, 64, device="cuda", dtype=BF)
    o, lse = lasad.lasad_forward_window(q, k, k, 4, want_lse=True)
    assert o.shape == q.shape and lse.shape == (2, 4, 0)
    g = lasad.lasad_backward_window(q, k, k, o, lse, q, 4, 1)
    assert (g[1] == 0).all() and (g[2] == 0).all() and g[0].shape == q.shape
    q, k = torch.ones(2, 5, 4, 64, device="cuda", dtype=F), torch.empty(2, 0, 2, 64, device="cuda", dtype=F)
    o, lse = lasad.lasad_forward_window(q, k, k, 4, 2, want_lse=True)
    assert (o == 0).all() and (lse == -float("inf")).all()
    g = lasad.lasad_backward_window(q, k, k, o, lse, q, 4, 2)
    assert (g[0] == 0).all() and g[1].shape == k.shape


@pytest.mark.parametrize("split", [40, 64, 97])
def test_two_calls_are_one(lasad, split):
    """A sequence in two calls (the second from start_pos on, against all keys) is the sequence in one, bit for bit where tiles
    are met in the same order and within the bound elsewhere."""
    c = (F, F, 64, 2, 1, 1, 0, 150, 150, 37, 2, None)
    q, k, v, mask = inputs(c)
    dev = [t.cuda() for t in (q, k, v)]
    a = lasad.lasad_forward_window(dev[0][:, :split], dev[1][:, :split], dev[2][:, :split], 37, 2)
    b = lasad.lasad_forward_window(dev[0][:, split:], dev[1], dev[2], 37, 2, start_pos=split)
    x = [t.double() for t in (q, k, v)]
    want, lse = ref.window_forward(*x, mask, 0.125)
    check(torch.cat((a, b), 1), want, ref.window_forward_bounds(*x, mask, 0.125, F, F, want, lse)[0], "o")


# ---- single tokens -----------------------------------------------------------------------------------------------

# dtype, out dtype, d, Hq, Hk, window, sinks, rows of the cache
STEPS = [(BF, BF, 64, 4, 4, 16, 1, 17), (BF, F, 64, 6, 2, 20, 4, 24), (F, F, 64, 5, 1, 7, 0, 7), (F, F, 32, 4, 2, 16, 3, 40),
         (BF, BF, 128, 8, 1, 9, 2, 11), (F, F, 128, 3, 1, 1, 0, 1), (BF, F, 32, 4, 1, 1, 5, 6), (BF, BF, 64, 2, 1, 2 ** 31 - 1, 3, 64)]


@pytest.mark.parametrize("c", STEPS, ids=lambda c: f"{str(c[0])[6:]}-{str(c[1])[6:]}-d{c[2]}-{c[3]}x{c[4]}-w{c[5]}-s{c[6]}-rows{c[7]}")
def test_steps_walk_a_sequence_through_the_cache(lasad, c):
    dt, ot, d, Hq, Hk, w, s, rows = c
    B, N = 2, 60
    q, k, v = ref.draw((B, N, Hq, d), dt, 1), ref.draw((B, N, Hk, d), dt, 2), ref.draw((B, N, Hk, d), dt, 3)
    kc, vc = (torch.full((B, Hk, rows, d), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    outs = []
    for t in range(N):
        outs.append(lasad.lasad_decode_step_window(*(x[:, t].contiguous().cuda() for x in (q, k, v)), kc, vc, t, w, s, out_dtype=ot))
    mask = ref.seen_mask(N, N, 0, w, s, None, B)
    x = [t.double() for t in (q, k, v)]
    want, lse = ref.window_forward(*x, mask, d ** -0.5)
    # (fp32 arithmetic whatever the storage type: no rounded operand)
    check(torch.stack(outs, 1), want, ref.window_forward_bounds(*x, mask, d ** -0.5, F, ot, want, lse)[0], "o")
    for cache, x in ((kc, k), (vc, v)):
        last = {ref.cache_row(j, s, rows): j for j in range(N)}
        for r in range(rows):
            got = cache[:, :, r].cpu()
            assert torch.equal(got, x[:, last[r]]) if r in last else got.isnan().all()


@pytest.mark.parametrize("dtype,G,d", [(BF, 1, 64), (BF, 2, 128), (F, 3, 64), (BF, 4, 32), (BF, 5, 64), (F, 9, 32)])
def test_steps_with_a_position_for_every_row(lasad, dtype, G, d):
    B, Hk, w, s, rows = 7, 2, 24, 3, 30
    pos = torch.tensor([0, 2, 26, 29, 500, -1, 2 ** 30], dtype=torch.int32)
    q, k, v = ref.draw((B, Hk * G, d), dtype, 1).cuda(), ref.draw((B, Hk, d), dtype, 2).cuda(), ref.draw((B, Hk, d), dtype, 3).cuda()
    caches = [ref.draw((B, Hk, rows, d), dtype, i).cuda() for i in (4, 5)]
    one = [c.clone() for c in caches]
    out = torch.full_like(q, 9.0)
    got = lasad.lasad_decode_step_window(q, k, v, *caches, pos.cuda(), w, s, out=out)
    for b in range(B):
        p = int(pos[b])
        part = [c[b:b + 1].clone() for c in one]
        if p < 0:
            assert (got[b] == 9.0).all()
        else:
            want = lasad.lasad_decode_step_window(q[b:b + 1], k[b:b + 1], v[b:b + 1], *part, p, w, s)
            assert torch.equal(got[b], want[0])
        assert all(torch.equal(c[b], x[0]) for c, x in zip(caches, part))
    # a cache with no room to go round: a position behind its end is inactive
    caches = [c.clone() for c in one]
    out.fill_(9.0)
    got = lasad.lasad_decode_step_window(q, k, v, *caches, pos.cuda(), 28, s, out=out)
    for b in range(B):
        assert (got[b] == 9.0).all() == (not 0 <= int(pos[b]) < rows)
    assert torch.equal(caches[0][4:], one[0][4:])


@pytest.mark.parametrize("dtype,d,G,count,pos", [(BF, 64, 1, 3001, 3000), (BF, 64, 3, 2500, 9999), (F, 128, 1, 1700, 1699), (F, 32, 2, 5000, 70000)])
def test_long_windows_over_several_workgroups(lasad, dtype, d, G, count, pos):
    B, Hk, s = 1, 2, 64
    w = rows = count
    rows += s
    q, k, v = ref.draw((B, Hk * G, d), dtype, 1), ref.draw((B, Hk, d), dtype, 2), ref.draw((B, Hk, d), dtype, 3)
    kc, vc = ref.draw((B, Hk, rows, d), dtype, 4), ref.draw((B, Hk, rows, d), dtype, 5)
    assert lasad.lasad_decode_step_window_workspace_bytes(B, Hk * G, Hk, d, rows, w, s) > 0
    dev = [t.cuda() for t in (kc, vc)]
    got = lasad.lasad_decode_step_window(q.cuda(), k.cuda(), v.cuda(), *dev, pos, w, s, out_dtype=F)
    alone = lasad.lasad_decode_step_window(q.cuda(), k.cuda(), v.cuda(), *dev, pos, w, s, out_dtype=F, use_workspace=False)
    js = [j for j in range(pos + 1) if pos - j < w or j < s]
    at = [ref.cache_row(j, s, rows) for j in js]
    kc[:, :, at[-1]], vc[:, :, at[-1]] = k, v
    x = [q[:, None].double(), kc[:, :, at].transpose(1, 2).double(), vc[:, :, at].transpose(1, 2).double()]
    mask = torch.ones(B, 1, len(js), dtype=torch.bool)
    want, lse = ref.window_forward(*x, mask, d ** -0.5)
    bound = ref.window_forward_bounds(*x, mask, d ** -0.5, F, F, want, lse)[0]
    check(got[:, None], want, bound, "o")
    check(alone[:, None], want, bound, "o without a workspace")


def test_a_step_reads_no_row_that_it_does_not_see(lasad):
    B, Hk, d, w, s, rows = 1, 2, 64, 40, 2, 100
    q, k, v = ref.draw((B, 2, d), BF, 1).cuda(), ref.draw((B, Hk, d), BF, 2).cuda(), ref.draw((B, Hk, d), BF, 3).cuda()
    kc, vc = ref.draw((B, Hk, rows, d), BF, 4).cuda(), ref.draw((B, Hk, rows, d), BF, 5).cuda()
    want = lasad.lasad_decode_step_window(q, k, v, kc.clone(), vc.clone(), 70, w, s)
    hidden = [r for r in range(rows) if not (r < s or 31 <= r < 70)]
    kc[:, :, hidden], vc[:, :, hidden] = float("nan"), float("nan")
    assert torch.equal(lasad.lasad_decode_step_window(q, k, v, kc, vc, 70, w, s), want)


def test_another_stream_and_graph_replays(lasad):
    c = CASES[1]
    q, k, v = (t.cuda() for t in inputs(c)[:3])
    do = ref.draw(q.shape, BF, 5).cuda()
    w, s, start = c[9], c[10], c[6]
    kc, vc = (ref.draw((2, 2, 2600, 64), BF, i).cuda() for i in (8, 9))
    q1, k1 = q[:, 0].contiguous(), k[:, 0].contiguous()

    def run(stream=None):
        o, lse = lasad.lasad_forward_window(q, k, v, w, s, start_pos=start, want_lse=True, stream=stream)
        g = lasad.lasad_backward_window(q, k, v, o, lse, do, w, s, start_pos=start, stream=stream)
        return (o, lse, *g, lasad.lasad_decode_step_window(q1, k1, k1, kc, vc, 5000, 2500, 100, stream=stream))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        q.copy_(ref.draw(q.shape, BF, 90 + i))
        q1.copy_(q[:, 1])
        want = run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
