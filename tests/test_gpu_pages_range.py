"""Attention over the paged 8-bit cache where keys or values are far from 1: sums of P v that would pass fp32 although the average does not,
keys whose scale times the attention's is subnormal."""
import pytest
import torch

import pages_reference as pr
import softmax_layer_reference as ref
from test_gpu_pages import BF, EPS, F, LAST, cpu, expected, lasad, on_gpu, packed, project, query_bound, spoil, table_of  # noqa: F401

pytestmark = pytest.mark.gpu

TOP = 3.0e38                                               # the largest value (bf16 and fp32 reach 3.38e38)
# Terms below 2^-84 of a row's largest may count as 0 beside values from 2^72 on (P is held 2^42 lower there): times 2^14 keys
LOST = 2.0 ** (14 - 84) * TOP


def lift_values(pages, table, which, sign):
    """The pages `which` of every row (by their number in it; None: all) as large as fp32 allows, of one sign (`sign`) or of both."""
    for b in range(table.shape[0]):
        for j in range(table.shape[1]):
            page = int(table[b, j])
            if page < 0 or (which is not None and j not in which):
                continue
            if sign:
                pages.v.view(torch.uint8)[page] &= 0x7f
            pages.v_scales[page] = TOP / pr.TOP


# dtype, out dtype, d, Hq, Hk, lengths, positions, window, sinks
SHAPES = [
    (BF, BF, 64, 24, 24, [1000, 920], [30, 0], 900, 70),   # two tiles of columns a wavefront
    (BF, F, 32, 4, 2, [150, 300], [700, 0], 900, 0),       # one
    (F, F, 64, 4, 2, [90], [700], 2 ** 30, 0),
    (BF, BF, 128, 4, 1, [150], [700], 800, 3),
    (F, F, 128, 2, 2, [70], [900], 2 ** 30, 0),
    (BF, BF, 64, 4, 2, [7, 1], [700, 900], 2 ** 30, 0),    # wavefronts over the pages
    (BF, F, 64, 2, 2, [3, 1], [5000, 4000], 4500, 8),      # and workgroups
    (F, F, 32, 4, 4, [1, 1], [4000, 3000], 2 ** 30, 0),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
@pytest.mark.parametrize("which", [None, (3,), (0, 1, 7)])
@pytest.mark.parametrize("sign", [True, False])
def test_large_values(lasad, case, which, sign):
    """Flat weights (small queries), so that many values of the largest size are averaged."""
    dt, odt, d, Hq, Hk, lengths, positions, window, sinks = SHAPES[case]
    one = all(n == 1 for n in lengths)
    rows = packed(lengths, positions)
    T = sum(lengths)
    need = sum((p + n + 63) // 64 for _, n, p in rows)
    table = table_of(rows, need, 8)
    pages = pr.filled_pool(lasad, need, Hk, d, 12)
    lift_values(pages, table, which, sign)
    spoil(pages, table, rows)
    q = ref.draw((T, Hq, d), dt, 30 + case, 0.1).cuda()
    t, pos, starts = on_gpu(table, rows, one)
    o = lasad.lasad_forward_pages(q, pages, t, pos, window, sinks, row_starts=starts, out_dtype=odt).cpu().double()
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, window, sinks, d ** -0.5, dt, odt)
    assert ((o - want).abs() <= bound + (LOST if (want.abs() > 1e20).any() else 0.0)).all()


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("lengths", [[300], [3], [1]])
@pytest.mark.parametrize("kind", range(3))
def test_large_values_and_scores_that_move_the_maximum(lasad, dt, lengths, kind):
    """Scores that rise from page to page, jump by hundreds, or fall, before and behind a page of large values."""
    d, Hq, Hk, p, window = 64, 4, 2, 700, 2 ** 30
    rows = packed(lengths, [p])
    table = table_of(rows, 20, 8)
    pages = pr.filled_pool(lasad, 20, Hk, d, 12)
    lift_values(pages, table, (3, 6), False)
    for j in range(table.shape[1]):
        if table[0, j] >= 0:
            pages.k_scales[int(table[0, j])] *= 2.0 ** (0.5 * j, 9.0 if j in (2, 5, 9) else 0.0, -0.5 * j)[kind]
    q = ref.draw((sum(lengths), Hq, d), dt, 3).cuda()
    t, pos, starts = on_gpu(table, rows, lengths == [1])
    o = lasad.lasad_forward_pages(q, pages, t, pos, window, 0, row_starts=starts).cpu().double()
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, window, 0, d ** -0.5, dt, dt)
    # what a maximum that moves leaves out is as small beside that maximum's own term
    assert ((o - want).abs() <= bound + LOST).all()


# dtype, d, Hq, Hk, positions, window
STEPS = [
    (BF, 64, 6, 2, [63, 640, 1000, 5], 2 ** 30),
    (BF, 64, 12, 2, [640, 1000], 900),
    (F, 64, 40, 2, [640, 1000], 2 ** 30),
    (F, 32, 4, 4, [640, 100], 2 ** 30),
    (BF, 128, 4, 2, [640, 1000], 2 ** 30),
    (BF, 64, 2, 2, [5000, 4100], 2 ** 30),
]


@pytest.mark.parametrize("case", range(len(STEPS)))
@pytest.mark.parametrize("which", [None, (3,)])
def test_large_values_in_steps(lasad, case, which):
    dt, d, Hq, Hk, positions, window = STEPS[case]
    rows = [(b, 1, p) for b, p in enumerate(positions)]
    B, grid = len(rows), (100, 100)
    need = sum(p // 64 + 1 for p in positions)
    table = table_of(rows, need, 8)
    pages = pr.filled_pool(lasad, need, Hk, d, 12)
    lift_values(pages, table, which, True)
    q, k, v = (t.contiguous() for t in project(B, Hq, Hk, d, dt, 50 + case))
    q, v = q * 0.1, (v.abs() * 1e37 if which is None else v)
    before = cpu(pages)
    t, pos, _ = on_gpu(table, rows)
    yk, ek = expected(k, None, rows, B, grid[1], 2, False, -1.0, dt)
    yq, eq = expected(q, None, rows, B, grid[1], 2, False, -1.0, dt)
    o = lasad.lasad_decode_step_pages(q, k, v, pages, t, pos, *grid, window, norm_eps=-1.0).cpu().double()
    pr.check_append(before, cpu(pages), table, rows, 10000, yk, ek, v.cpu().double())
    want, bound = pr.attend(yq, cpu(pages), table, rows, LAST, window, 0, d ** -0.5, dt, dt)
    bound = bound + query_bound(yq, eq, cpu(pages), table, rows, window, 0, d ** -0.5, dt)
    assert ((o - want).abs() <= bound + LOST).all()


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("lengths", [[200], [3], [1]])
def test_small_keys(lasad, dt, lengths):
    """Keys of 2^-126, held with the least scale, against queries of 2^120: scores of some tenths, from a product of scales below 2^-126."""
    d, Hq, Hk, p, scale = 64, 4, 2, 300, 0.125
    T, m = sum(lengths), p + sum(lengths)
    rows = packed(lengths, [p])
    table = table_of(rows, 10, 8)
    pages = pr.new_pool(lasad, 10, Hk, d)
    k = (ref.draw((m, Hk, d), torch.float64, 5) * 2.0 ** -125).to(F).cuda()
    v = ref.draw((m, Hk, d), F, 6).cuda()
    starts = torch.tensor([0, m], dtype=torch.int32).cuda()
    lasad.lasad_append_pages(None, k, v, pages, table.cuda(), 0, 32, 32, norm_eps=-1.0, rope=0, row_starts=starts)
    assert (pages.k_scales[table[0, 0].item()] == 2.0 ** -126).all()
    q = (ref.draw((T, Hq, d), torch.float64, 7) * 2.0 ** 120).to(dt).cuda()
    t, pos, starts = on_gpu(table, rows, lengths == [1])
    o = lasad.lasad_forward_pages(q, pages, t, pos, 2 ** 30, 0, row_starts=starts, scale=scale).cpu().double()
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, 2 ** 30, 0, scale, dt, dt)
    # the product of the scales, 2^-128.5, is rounded by up to 2^-150: 2^-21 of a score; scores below 1
    kk, vv = pr.values(cpu(pages))
    slack = torch.expm1(torch.tensor(2 * 2.0 ** -21)) * vv[torch.isfinite(vv)].abs().max()
    assert ((o - want).abs() <= bound + slack).all()
