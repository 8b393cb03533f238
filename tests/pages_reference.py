"""The paged 8-bit cache in 64 bits (torch on the CPU): what pages hold, what an append may leave in them, attention over them.

Bounds: those of softmax_layer_reference, with one rounding to e4m3 for what is stored: half a step, 2^-4 of the value, and 2^-10 scales
below the smallest normal code."""
import math

import torch

import softmax_layer_reference as ref

PAGE, TOP = 64, 448.0
U = ref.U
PLACE = torch.tensor([16 * (t // 4 % 4) + 4 * (t // 16) + t % 4 for t in range(PAGE)])       # of a position in a page of v


def codes(pages):
    """k and v of a pool in the order of positions, [n_pages, Hk, 64, d] in fp64, without their scales."""
    k, v = pages[0].cpu().double(), pages[1].cpu().double()
    return k, v[..., PLACE].transpose(2, 3)


def values(pages):
    k, v = codes(pages)
    return k * pages[2].cpu().double()[:, :, None, None], v * pages[3].cpu().double()[:, :, None, None]


def new_pool(lasad, n_pages, Hk, d, device="cuda"):
    """Pages as a pool may hold them before anything is written: NaN."""
    pages = lasad.new_pages(n_pages, Hk, d, device)
    for t in pages[:2]:
        t.view(torch.uint8).fill_(0x7f)
    for t in pages[2:]:
        t.fill_(math.nan)
    return pages


def filled_pool(lasad, n_pages, Hk, d, seed, spread=1.0, device="cuda"):
    """Pages of normal numbers, the scales of different pages apart."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for width in (d, d):
        x = torch.randn(n_pages, Hk, PAGE, width, generator=gen)
        scale = x.abs().amax((2, 3)) / TOP
        out.append(((x / scale[..., None, None]).to(torch.float8_e4m3fn), scale * spread ** torch.randn(n_pages, Hk, generator=gen)))
    (k, ks), (v, vs) = out
    at = torch.empty(PAGE, dtype=torch.long)
    at[PLACE] = torch.arange(PAGE)
    v = v.view(torch.uint8).transpose(2, 3)[..., at].contiguous().view(torch.float8_e4m3fn)
    return lasad.Pages(*(t.to(device) for t in (k, v, ks.float(), vs.float())))


def rows_of(starts, pos, B, T):
    """(first token, tokens, position) of every row."""
    if starts is None:
        return [(b, 1, pos[b]) for b in range(B)]
    return [(starts[b], starts[b + 1] - starts[b], pos[b]) for b in range(B)]


def active(row, table, last_pos):
    first, n, p = row
    return n > 0 and p >= 0 and p + n <= min(last_pos, table.shape[1] * PAGE)


def check_stored(y, e, old_codes, old_scale, new_codes, new_scale, begin, what):
    """One head of one page: y [n, d] the call's numbers in fp64, off by at most e in the kernel, from position `begin` on; codes [64, d] before
    and after the call."""
    n = y.shape[0]
    fine = torch.isfinite(y)
    most = y[fine].abs().max().item() if fine.any() else 0.0
    slack = e[fine].max().item() if fine.any() else 0.0
    old = old_scale if begin > 0 else 0.0
    if old > 0:
        power = new_scale / old
        assert math.log2(power) == int(math.log2(power)) and power >= 1, what
        assert most - slack <= TOP * new_scale * (1 + 2 * U), what
        assert power == 1 or most + slack > TOP * new_scale / 2 * (1 - 2 * U), what
        kept = (old_codes[:begin].float() / power).to(torch.float8_e4m3fn).double()
        assert torch.equal(new_codes[:begin].nan_to_num(999.0), kept.nan_to_num(999.0)), what
    else:
        # (a division: half a step; a subnormal quotient is not below the least scale)
        want = max(most / TOP, 2.0 ** -126) if most > 0 else 0.0
        assert abs(new_scale - want) <= slack / TOP + 2 * U * want, (what, new_scale, want)
        if begin > 0:                                      # (a page whose tokens are all zero, or NaN)
            assert torch.equal(new_codes[:begin].nan_to_num(999.0), old_codes[:begin].nan_to_num(999.0)), what
    got = new_codes[begin:begin + n]
    assert torch.equal(torch.isnan(got), ~fine), what
    value = got * new_scale
    # half a step of e4m3; the quotient is a rounding or two off, which the numbers' own bound has beside it
    allowed = torch.maximum(y.abs() * 2.0 ** -4 * (1 + 4 * U), torch.tensor(2.0 ** -10 * new_scale)) + e + 4 * U * y.abs()
    assert ((value - y).abs() <= allowed)[fine].all(), (what, ((value - y).abs() / allowed)[fine].max().item())
    assert (got[fine].abs() <= TOP).all(), what


def check_append(before, after, table, rows, last_pos, k, k_error, v):
    """Pools before and after a call (on the CPU); k, v [T, Hk, d] what was to be stored, in fp64.  Nothing else has changed."""
    zero = torch.zeros_like(v)
    old, new = codes(before), codes(after)
    touched = [torch.zeros(t.shape, dtype=torch.bool) for t in old]
    scaled = torch.zeros(before[2].shape, dtype=torch.bool)
    for b, row in enumerate(rows):
        if not active(row, table, last_pos):
            continue
        first, n, p = row
        for j in range(p // PAGE, (p + n - 1) // PAGE + 1):
            page = int(table[b, j])
            if not 0 <= page < before[0].shape[0]:
                continue
            lo, hi = max(p, j * PAGE), min(p + n, (j + 1) * PAGE)
            tokens = slice(first + lo - p, first + hi - p)
            begin = lo - j * PAGE
            for t in touched:
                t[page, :, :hi - j * PAGE] = True
            scaled[page] = True
            for h in range(k.shape[1]):
                for i, (y, e) in enumerate(((k, k_error), (v, zero))):
                    check_stored(y[tokens, h], e[tokens, h], old[i][page, h], before[2 + i][page, h].item(), new[i][page, h],
                                 after[2 + i][page, h].item(), begin, f"row {b} page {j} head {h} {'kv'[i]}")
    for i in range(2):
        left = ~touched[i]
        assert torch.equal(old[i][left].nan_to_num(999.0), new[i][left].nan_to_num(999.0))
        assert torch.equal(before[2 + i][~scaled].nan_to_num(999.0), after[2 + i][~scaled].nan_to_num(999.0))


def attend(q, pages, table, rows, last_pos, window, sinks, scale, dtype, out_dtype):
    """q [T, Hq, d] in fp64; the pool on the CPU.  Returns o and its bound, NaN rows' bound 0; both 0 where nothing is written."""
    kk, vv = values(pages)
    o, bound = torch.zeros_like(q), torch.zeros_like(q)
    for b, row in enumerate(rows):
        if not active(row, table, last_pos):
            continue
        first, n, p = row
        mask = ref.seen_mask(n, p + n, p, window, sinks)
        k, v = (torch.zeros(1, p + n, x.shape[1], x.shape[3], dtype=torch.float64) for x in (kk, vv))
        for j in range((p + n + PAGE - 1) // PAGE):
            page, m = int(table[b, j]), min(PAGE, p + n - j * PAGE)
            if 0 <= page < kk.shape[0]:
                k[0, j * PAGE:j * PAGE + m] = kk[page, :, :m].transpose(0, 1)
                v[0, j * PAGE:j * PAGE + m] = vv[page, :, :m].transpose(0, 1)
            else:
                mask[:, :, j * PAGE:(j + 1) * PAGE] = False
        used = mask[0].any(0)                              # what nobody sees may be anything
        k[0, ~used], v[0, ~used] = 0.0, 0.0
        x = q[None, first:first + n]
        got, lse = ref.window_forward(x, k, v, mask, scale)
        limit, _ = ref.window_forward_bounds(x, k, v, mask, scale, dtype, out_dtype, got, lse)
        o[first:first + n], bound[first:first + n] = got[0], limit[0]
    return o, bound


def written(rows, table, last_pos, T):
    """Which tokens belong to an active row."""
    on = torch.zeros(T, dtype=torch.bool)
    for row in rows:
        if active(row, table, last_pos):
            on[row[0]:row[0] + row[1]] = True
    return on
