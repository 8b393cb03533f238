"""64-bit references of the softmax layers' operators (torch on the CPU; gradients by automatic differentiation), and the
error bounds of the tests that use them.

Bounds: u = 2^-24 is the rounding of one fp32 operation.  They count the roundings on the longest path to a result and
multiply them with the magnitudes that pass through it, so that cancellation is allowed for and nothing else; a result
stored in bf16 may be off by 2^-8 of its value on top."""
import math

import torch

U = 2.0 ** -24


def stored(dtype, value):
    """What storing `value` (fp64) in dtype may add to its error."""
    return (2.0 ** -8 if dtype == torch.bfloat16 else U) * value.abs()


def draw(shape, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(dtype)


# ---- norms and rotation --------------------------------------------------------------------------------------------

def pair_channels(d, two_axes, halves):
    """Channels of the first and the second members, in the order of the pairs."""
    if not halves:
        return list(range(0, d, 2)), list(range(1, d, 2))
    span = d // 2 if two_axes else d
    first = [s + i for s in range(0, d, span) for i in range(span // 2)]
    return first, [i + span // 2 for i in first]


def angles(positions, d, grid_w, two_axes, base):
    """[.., d / 2] in fp64."""
    p = positions.double()[..., None]
    i = torch.arange(d // 2, dtype=torch.float64)
    if two_axes:
        axis = torch.where(i < d // 4, torch.div(p, grid_w, rounding_mode="floor"), p.remainder(grid_w))
        return axis * torch.exp(-(i % (d // 4)) / (d // 4) * math.log(base))
    return p * torch.exp(-i / (d // 2) * math.log(base))


def qk_row(x, w, positions, grid_w, rope, halves, base, eps):
    """x: [.., heads, d] fp64, positions: [..]; w [heads, d], [d] or None.  Returns y."""
    d = x.shape[-1]
    if eps >= 0:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w
    if rope == 0:
        return x
    a = angles(positions, d, grid_w, rope == 2, base)[..., None, :]
    lo, hi = pair_channels(d, rope == 2, halves)
    p, q = x[..., lo], x[..., hi]
    y = torch.empty_like(x)
    y[..., lo] = p * a.cos() - q * a.sin()
    y[..., hi] = p * a.sin() + q * a.cos()
    return y


def pair_size(x, rope, halves):
    """|a| + |b| of the pair that a channel belongs to (|x| without a rotation)."""
    if rope == 0:
        return x.abs()
    lo, hi = pair_channels(x.shape[-1], rope == 2, halves)
    s = x[..., lo].abs() + x[..., hi].abs()
    out = torch.empty_like(x)
    out[..., lo] = s
    out[..., hi] = s
    return out


FAR = 2.0 ** -50        # an angle in fp64, here and in the kernel: frequency and product are off by four roundings, 2^-51 of it


def qk_forward_bound(x, w, rope, halves, eps, out_dtype, y, last_pos=0):
    """Roundings on the way to y: 8 squares added in a lane and 4 additions over lanes (halved by the root), mean, root,
    two products: 12; the reduced angle and its cosine: 2^-22 = 4 u beside the value; product and sum: 2."""
    xh = qk_row(x, w, None, 1, 0, False, 2.0, eps)
    return (20 * U + FAR * last_pos) * pair_size(xh, rope, halves) + stored(out_dtype, y)


def qk_backward_reference(x, w, dy, positions, grid_w, rope, halves, base, eps):
    x = x.detach().clone().requires_grad_()
    w = None if w is None else w.detach().clone().requires_grad_()
    qk_row(x, w, positions, grid_w, rope, halves, base, eps).backward(dy)
    return x.grad, None if w is None else w.grad


def qk_backward_bound(x, w, dy, rope, halves, eps, grad_dtype, dx, last_pos=0):
    """Bounds of dx and of one head's term of dw: the gradient turned back (4 for the angles, 2 operations) times w is off by 8
    roundings, the sums over the row by 12 more, the norm's factor by 12; the three products and the difference add 5."""
    g = pair_size(dy, rope, halves) * (1 + FAR * last_pos / (24 * U))
    if eps < 0:
        return 8 * U * g + stored(grad_dtype, dx), None
    rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh = (x * rstd).abs()
    gw = g if w is None else g * w.abs()
    m = (gw * xh).mean(-1, keepdim=True)
    return 48 * U * rstd * (gw + xh * m) + stored(grad_dtype, dx), 24 * U * g * xh


# ---- attention with a window and sinks -----------------------------------------------------------------------------

def seen_mask(n, m, start, window, sinks, lens=None, B=1):
    """[B, n, m]: does query i (position start + i) of a batch row see key j?"""
    p, j = start + torch.arange(n)[:, None], torch.arange(m)[None]
    seen = ((j <= p) & ((p - j < window) | (j < sinks)))[None].expand(B, n, m)
    if lens is not None:
        seen = seen & (j[None] < torch.as_tensor(lens).view(B, 1, 1))
    return seen


def shared(x, Hq):
    """Key heads repeated for the query heads that share them: [B, m, Hk, d] -> [B, m, Hq, d]."""
    return x.repeat_interleave(Hq // x.shape[2], 2)


def window_forward(q, k, v, mask, scale):
    """q [B, n, Hq, d], k, v [B, m, Hk, d] in fp64, mask [B, n, m].  Returns o and lse [B, Hq, n]."""
    k, v = shared(k, q.shape[2]), shared(v, q.shape[2])
    s = torch.einsum("bihd,bjhd->bhij", q, k) * scale
    s = s.masked_fill(~mask[:, None], -math.inf)
    lse = torch.logsumexp(s, -1) if s.shape[-1] else s.new_full(s.shape[:-1], -math.inf)
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
    return torch.einsum("bhij,bjhd->bihd", p, v), lse


def window_backward(q, k, v, do, mask, scale):
    """The formulas of the gradients, nothing of them by automatic differentiation (a CPU test compares the two)."""
    Hk, Hq = k.shape[2], q.shape[2]
    o, lse = window_forward(q, k, v, mask, scale)
    ks, vs = shared(k, Hq), shared(v, Hq)
    s = torch.einsum("bihd,bjhd->bhij", q, ks) * scale
    p = torch.where(mask[:, None], torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None]), 0.0)
    dp = torch.einsum("bihd,bjhd->bhij", do, vs)
    ds = p * (dp - (do * o).sum(-1).transpose(1, 2)[..., None]) * scale
    fold = lambda x: x.unflatten(2, (Hk, Hq // Hk)).sum(3)
    return (torch.einsum("bhij,bjhd->bihd", ds, ks), fold(torch.einsum("bhij,bihd->bjhd", ds, q)),
            fold(torch.einsum("bhij,bihd->bjhd", p, do)))


def _rounded(dtype):
    """Rounding of a matrix-core operand formed by the kernel."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else 0.0


def _score_errors(q, k, mask, scale, s_abs_max=None):
    """[B, Hq, n]: bound of the error of any seen score of a query (as a power's exponent), and how many keys it sees."""
    a = torch.einsum("bihd,bjhd->bhij", q.abs(), shared(k, q.shape[2]).abs()) * scale
    a = a.masked_fill(~mask[:, None], 0.0)
    top = a.amax(-1) if a.shape[-1] else a.new_zeros(a.shape[:-1])
    # d products added up; scaled, shifted, exponential: 8 roundings of numbers no larger than the largest sum
    return (q.shape[-1] + 8) * U * (top + 1), mask.sum(-1)[:, None].expand(top.shape)


def window_forward_bounds(q, k, v, mask, scale, dtype, out_dtype, o, lse):
    """A term is off by the score's error, the sum by as much, both by one rounding an addition and a rescaling (at most two a
    key); bf16: the term is rounded to the operand's type."""
    e, count = _score_errors(q, k, mask, scale)
    pv, _ = window_forward(q, k, v.abs(), mask, scale)
    rel = 2 * e + (4 * count + 16) * U + _rounded(dtype)
    lse_bound = e + (2 * count + 16) * U + 4 * U * lse.masked_fill(lse == -math.inf, 0.0).abs()
    return pv * rel.transpose(1, 2)[..., None] + stored(out_dtype, o), lse_bound


def window_backward_bounds(q, k, v, do, mask, scale, dtype, grad_dtype, grads):
    """P is off by the score's error and that of lse; dP by its d products; delta by its d products and by o's error, storing
    included; dS by all of these and its rounding as an operand; a sum by one rounding an addition."""
    Hk, Hq, d = k.shape[2], q.shape[2], q.shape[3]
    ks, vs = shared(k, Hq), shared(v, Hq)
    o, lse = window_forward(q, k, v, mask, scale)
    e, count = _score_errors(q, k, mask, scale)
    o_bound, lse_bound = window_forward_bounds(q, k, v, mask, scale, dtype, dtype, o, lse)
    s = torch.einsum("bihd,bjhd->bhij", q, ks) * scale
    p = torch.where(mask[:, None], torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None]), 0.0)
    dp = torch.einsum("bihd,bjhd->bhij", do, vs)
    g = torch.einsum("bihd,bjhd->bhij", do.abs(), vs.abs())
    delta = (do * o).sum(-1).transpose(1, 2)[..., None]
    delta_bound = ((do.abs() * o_bound).sum(-1) + d * U * (do * o).abs().sum(-1)).transpose(1, 2)[..., None]
    p_rel = (e + lse_bound + 8 * U)[..., None]
    x = p * (dp - delta).abs()
    ds_err = (x * (p_rel + 4 * U + _rounded(dtype)) + p * ((d + 2) * U * g + delta_bound + 2 * U * delta.abs())) * scale
    ds_abs = x * scale
    fold = lambda t: t.unflatten(2, (Hk, Hq // Hk)).sum(3)
    keys = (count.amax() + 16) * U
    queries = ((mask.sum(1).amax() if mask.numel() else 0) * (Hq // Hk) + 80) * U
    dq = torch.einsum("bhij,bjhd->bihd", ds_err + keys * ds_abs, ks.abs())
    dk = fold(torch.einsum("bhij,bihd->bjhd", ds_err + queries * ds_abs, q.abs()))
    dv = fold(torch.einsum("bhij,bihd->bjhd", p * (p_rel + queries + _rounded(dtype)), do.abs()))
    return [b + stored(grad_dtype, t) for b, t in zip((dq, dk, dv), grads)]


def cache_row(j, sinks, rows):
    return j if j < sinks else sinks + (j - sinks) % (rows - sinks)
