"""Attention of bf16 queries over the paged 8-bit cache with fp32 results: P is not rounded to bf16."""
import pytest
import torch

import pages_reference as pr
import softmax_layer_reference as ref
from test_gpu_pages import BF, F, LAST, cpu, lasad, on_gpu, packed, spoil, table_of  # noqa: F401

pytestmark = pytest.mark.gpu

# d, Hq, Hk, lengths, positions, window, sinks
CASES = [
    (64, 24, 24, [1000, 920], [30, 0], 500, 70),           # two tiles of columns a wavefront
    (32, 26, 26, [1000, 920], [30, 0], 500, 70),
    (64, 4, 2, [150, 64], [61, 300], 96, 16),              # one
    (32, 4, 4, [100, 2], [7, 62], 64, 1),
    (128, 4, 2, [70, 64, 9], [3, 0, 500], 77, 4),
    (128, 8, 4, [1000, 920], [30, 0], 500, 70),
    (64, 6, 2, [3, 1, 4], [700, 64, 900], 800, 2),         # wavefronts over the pages
    (32, 4, 1, [3, 1], [700, 64], 800, 0),
    (128, 8, 1, [1, 1], [3000, 2900], 2800, 70),           # and workgroups
    (64, 2, 2, [3, 1], [5000, 4000], 4500, 8),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_fp32_results_of_bf16_queries(lasad, case):
    d, Hq, Hk, lengths, positions, window, sinks = CASES[case]
    rows = packed(lengths, positions)
    T = sum(lengths)
    need = sum((p + n + 63) // 64 for _, n, p in rows)
    table = table_of(rows, need, 8)
    pages = pr.filled_pool(lasad, need, Hk, d, 12, spread=1.5)
    spoil(pages, table, rows)
    q = ref.draw((T, Hq, d), BF, 30 + case).cuda()
    t, pos, starts = on_gpu(table, rows)
    o = lasad.lasad_forward_pages(q, pages, t, pos, window, sinks, row_starts=starts, out_dtype=F).cpu().double()
    want, bound = pr.attend(q.cpu().double(), cpu(pages), table, rows, LAST, window, sinks, d ** -0.5, F, F)
    # two bf16 parts of P leave out half a step of the second, 2^-9 of a number below 2^-8 of P: 2^-17; numerator and denominator of it
    size, _ = pr.attend(q.cpu().double(), [*cpu(pages)[:1], cpu(pages)[1].view(torch.uint8).bitwise_and(0x7f).view(torch.float8_e4m3fn), *cpu(pages)[2:]],
                        table, rows, LAST, window, sinks, d ** -0.5, F, F)
    assert ((o - want).abs() <= bound + 2 * 2.0 ** -17 * size).all(), ((o - want).abs() / bound).max().item()
