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
