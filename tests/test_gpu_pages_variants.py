"""Every kernel of the paged 8-bit cache that a call can choose, against the 64-bit reference: types, head dims, pairings, copies of few heads,
columns of a workgroup, splits and their join; pages enough that a wavefront's loop over whole ones goes round several times; pages
whose scales have to grow for the new tokens."""
import pytest
import torch

import pages_reference as pr
import softmax_layer_reference as ref
from test_gpu_pages import BASE, BF, EPS, F, LAST, cpu, cuda, expected, lasad, on_gpu, packed, project, query_bound, spoil, table_of, weights  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = [(BF, BF), (BF, F), (F, F)]


def lower(pages, by_k, by_v):
    pages.k_scales.mul_(by_k)
    pages.v_scales.mul_(by_v)


def grown(before, after, table, rows, last_pos, i):
    """The factors by which scales i (2: of keys, 3: of values) of the pages that had earlier tokens have grown."""
    out = []
    for b, row in enumerate(rows):
        if pr.active(row, table, last_pos) and row[2] % pr.PAGE:
            page = int(table[b, row[2] // pr.PAGE])
            out.append(after[i][page] / before[i][page])
    return torch.cat(out)


@pytest.mark.parametrize("dt, odt", TYPES)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("rope, halves", [(0, False), (2, False), (1, True), (2, True), (1, False)])
def test_append(lasad, dt, odt, d, rope, halves):
    Hq, Hk, lengths, positions, W = 3, 2, [70, 3, 1, 130, 20], [10, 60, 33, 64, 101], 23
    rows = packed(lengths, positions, lead=1)
    T = rows[-1][0] + rows[-1][1] + 1
    table = table_of(rows, 20, 3)
    wq, wk = weights(Hq, Hk, d, "heads")
    H = 250 // W + 1
    for by_k, by_v in ((0.125, 0.125), (0.125, 1.0), (1.0, 0.125)):
        pages = pr.filled_pool(lasad, 20, Hk, d, 11)
        lower(pages, by_k, by_v)
        before = cpu(pages)
        q, k, v = project(T, Hq, Hk, d, dt, 20)
        t, pos, starts = on_gpu(table, rows)
        mark = torch.full((T, Hq, d), 7.0, dtype=odt, device="cuda")
        lasad.lasad_append_pages(q, k, v, pages, t, pos, H, W, cuda(wq), cuda(wk), EPS, rope, int(halves), BASE, row_starts=starts, out=mark)
        yk, ek = expected(k, wk, rows, T, W, rope, halves, EPS, dt)
        now = cpu(pages)
        pr.check_append(before, now, table, rows, H * W, yk, ek, v.cpu().double())
        for i, by in ((2, by_k), (3, by_v)):
            if by < 1:
                assert (grown(before, now, table, rows, H * W, i) >= 2).all()
        yq, eq = expected(q, wq, rows, T, W, rope, halves, EPS, dt)
        on = pr.written(rows, table, H * W, T)
        got = mark.cpu().double()
        assert (got[~on] == 7.0).all()
        assert ((got - yq).abs() <= eq + ref.stored(odt, yq))[on].all()


# Hq, Hk, lengths, positions; how the launch has to be divided: columns of a workgroup, splits
FORWARDS = {
    "few": (6, 2, [4, 3, 1], [1400, 700, 63], 16, False),
    "split": (16, 8, [2, 1, 1, 1, 1, 1, 1], [7900, 700, 63, 64, 0, 130, 200], 16, True),
    "beside": (4, 2, [150, 64], [1400, 300], 64, False),
    "full": (26, 26, [1000, 900], [400, 0], 128, False),
}


def columns_taken(Hq, Hk, lengths, dt, d):
    G, T, B = Hq // Hk, sum(lengths), len(lengths)
    if T * G <= 32 * B:
        return 16
    return 128 if dt == BF and d <= 64 and (T * G // 128 + B) * Hk >= 384 else 64


@pytest.mark.parametrize("dt, odt", TYPES)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("kind", FORWARDS)
def test_attention(lasad, dt, odt, d, kind):
    Hq, Hk, lengths, positions, columns, split = FORWARDS[kind]
    if dt == F or d == 128:
        columns = min(columns, 64)
    assert columns_taken(Hq, Hk, lengths, dt, d) == columns
    window, sinks = 2 ** 30, 0
    rows = packed(lengths, positions)
    T, B = sum(lengths), len(rows)
    need = sum((p + n + 63) // 64 for _, n, p in rows)
    table = table_of(rows, need, 8)
    assert (lasad.lasad_forward_pages_workspace_bytes(B, Hq, Hk, d, T, False, table.shape[1], window, sinks) > 0) == split
    pages = pr.filled_pool(lasad, need, Hk, d, 12, spread=1.5)
    spoil(pages, table, rows)
    q = ref.draw((T, Hq, d), dt, 30).cuda()
    t, pos, starts = on_gpu(table, rows)
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, window, sinks, d ** -0.5, dt, odt)
    for use in (True, False) if split else (True,):
        o = lasad.lasad_forward_pages(q, pages, t, pos, window, sinks, row_starts=starts, out_dtype=odt, use_workspace=use).cpu().double()
        # (fp64 has exponentials that fp32 has not: 2^13 of them below 2^-126 of the largest, values below 2^4)
        assert ((o - want).abs() <= bound + 2.0 ** -109).all(), (use, ((o - want).abs() / bound).max().item())


@pytest.mark.parametrize("dt, odt", TYPES)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("G", [1, 3, 6, 12, 20])
@pytest.mark.parametrize("by_k, by_v", [(1.0, 1.0), (0.125, 0.125), (0.125, 1.0), (1.0, 0.125)])
def test_step(lasad, dt, odt, d, G, by_k, by_v):
    """New tokens in every block of 16 positions of their page, which is their wavefront's first, one behind others, or the row's only one;
    scales of keys and values that have to grow for them, both, one or none."""
    Hk, grid, window, sinks = 2, (50, 50), 2 ** 30, 0
    positions = [2100, 707, 1064, 63, 192 + 17, 39, 128, 384 + 5]
    rows = [(b, 1, p) for b, p in enumerate(positions)]
    B = len(rows)
    need = sum(p // 64 + 1 for p in positions)
    table = table_of(rows, need, 8)
    pages = pr.filled_pool(lasad, need, Hk, d, 12)
    lower(pages, by_k, by_v)
    spoil(pages, table, [(b, 1, p - 1) for b, p in enumerate(positions)])
    before = cpu(pages)
    q, k, v = (t.contiguous() for t in project(B, G * Hk, Hk, d, dt, 50))
    wq, wk = weights(G * Hk, Hk, d, "heads")
    t, pos, _ = on_gpu(table, rows)
    rope, halves = (2, False) if G % 2 else (1, True)
    yk, ek = expected(k, wk, rows, B, grid[1], rope, halves, EPS, dt)
    yq, eq = expected(q, wq, rows, B, grid[1], rope, halves, EPS, dt)
    assert lasad.lasad_decode_step_pages_workspace_bytes(B, G * Hk, Hk, d, table.shape[1], window, sinks) > 0
    for split in (True, False):
        mine = lasad.Pages(*(x.clone().cuda() for x in before))
        o = lasad.lasad_decode_step_pages(q, k, v, mine, t, pos, *grid, window, sinks, cuda(wq), cuda(wk), EPS, rope, int(halves), BASE,
                                          out_dtype=odt, use_workspace=split).cpu().double()
        now = cpu(mine)
        pr.check_append(before, now, table, rows, 2500, yk, ek, v.cpu().double())
        for i, by in ((2, by_k), (3, by_v)):
            if by < 1:
                assert (grown(before, now, table, rows, 2500, i) >= 2).all()
        want, bound = pr.attend(yq, now, table, rows, LAST, window, sinks, d ** -0.5, dt, odt)
        bound = bound + query_bound(yq, eq, now, table, rows, window, sinks, d ** -0.5, dt)
        assert ((o - want).abs() <= bound + 2.0 ** -112).all(), (split, ((o - want).abs() / bound).max().item())


@pytest.mark.parametrize("lengths, few", [([20, 12], True), ([20, 13], False), ([31, 1], True), ([63, 1], False), ([1, 64], False)])
@pytest.mark.parametrize("dt", [BF, F])
def test_attention_at_the_border_of_few_columns(lasad, lengths, few, dt):
    """32 columns a row on average, and one token more: wavefronts over the pages and splits, and neither."""
    d, Hq, Hk, positions, window = 32, 4, 2, [2000, 1900], 2 ** 30
    rows = packed(lengths, positions)
    T = sum(lengths)
    table = table_of(rows, 66, 8)
    assert (lasad.lasad_forward_pages_workspace_bytes(2, Hq, Hk, d, T, False, table.shape[1], window, 0) > 0) == few
    pages = pr.filled_pool(lasad, 66, Hk, d, 12, spread=1.5)
    spoil(pages, table, rows)
    q = ref.draw((T, Hq, d), dt, 30).cuda()
    t, pos, starts = on_gpu(table, rows)
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, window, 0, d ** -0.5, dt, dt)
    for use in (True, False):
        o = lasad.lasad_forward_pages(q, pages, t, pos, window, row_starts=starts, use_workspace=use).cpu().double()
        # (fp64 has exponentials that fp32 has not: 2^11 of them below 2^-126 of the largest, values below 2^4)
        assert ((o - want).abs() <= bound + 2.0 ** -111).all(), (use, ((o - want).abs() / bound).max().item())


@pytest.mark.parametrize("B, Hk, split", [(64, 2, True), (43, 3, False), (128, 1, True), (129, 1, False)])
def test_step_at_the_border_of_splits(lasad, B, Hk, split):
    """128 rows times key heads, the most that are split, and one more; a few long rows among short ones."""
    d, G, grid, window, dt = 32, 2, (50, 50), 2 ** 30, BF
    positions = [2100 if b in (0, B - 1) else (37 * b) % 150 for b in range(B)]
    rows = [(b, 1, p) for b, p in enumerate(positions)]
    need = sum(p // 64 + 1 for p in positions)
    table = table_of(rows, need, 8)
    assert (lasad.lasad_decode_step_pages_workspace_bytes(B, G * Hk, Hk, d, table.shape[1], window, 0) > 0) == split
    pages = pr.filled_pool(lasad, need, Hk, d, 12)
    before = cpu(pages)
    q, k, v = (t.contiguous() for t in project(B, G * Hk, Hk, d, dt, 50))
    t, pos, _ = on_gpu(table, rows)
    yk, ek = expected(k, None, rows, B, grid[1], 2, False, EPS, dt)
    yq, eq = expected(q, None, rows, B, grid[1], 2, False, EPS, dt)
    o = lasad.lasad_decode_step_pages(q, k, v, pages, t, pos, *grid, window).cpu().double()
    now = cpu(pages)
    pr.check_append(before, now, table, rows, 2500, yk, ek, v.cpu().double())
    want, bound = pr.attend(yq, now, table, rows, LAST, window, 0, d ** -0.5, dt, dt)
    bound = bound + query_bound(yq, eq, now, table, rows, window, 0, d ** -0.5, dt)
    assert ((o - want).abs() <= bound + 2.0 ** -112).all(), ((o - want).abs() / bound).max().item()
