"""Timed cases of the paged 8-bit cache of the softmax layers, in plain torch and through the framework's calls.

A server holds the keys and values of its images in pages of 64 positions, e4m3 codes with one scale for each page and key
head.  Three operators that belong together:

  append  the new tokens of every row (a prompt, the continuation of one, or one token): norm and rotation of the query and
          key heads, keys and values into the rows' pages.
  attend  attention of the new tokens' queries over the pages: causal, a window back and the first `sinks` positions.
  step    both for one token of every row.

A case is a dict of plain values:

  op            as above;  dtype  storage type of q, k, v and o ("bf16", "f32")
  B, Hq, Hk, d  rows, query heads, key heads (each shared by Hq / Hk query heads), channels of a head
  pos, n        position of a row's first new token, and how many new tokens it has (step: one);  ragged  rows are elsewhere, and
                have fewer tokens (some none)
  H, W          token grid;  rope, halves  "2d", "1d" or "none"; pairs (i, i + half) instead of (2i, 2i + 1)
  window, sinks (attend, step)

A page of k is [64 positions][d].  A page of v is [d][64]: position 16 b + 4 g + i of the page lies at 16 g + 4 b + i.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0
PAGE = 64
TOP = 448.0                  # the largest e4m3 value
LEAST = 2.0 ** -126          # the least scale of a page that is not all zeros


def listed():
    return [
        # One image sampled by the 12-head model: one token's heads and its page.  Launch and host latency.
        {"name": "append_one_image", "op": "append", "dtype": "bf16", "B": 1, "Hq": 12, "Hk": 12, "d": 64, "pos": 100, "n": 1,
         "ragged": False, "H": 16, "W": 16, "rope": "2d", "halves": False},
        # A batch of images of the base model, each continued from some rows of it that are given: pages begun in the middle.
        {"name": "append_base_continued", "op": "append", "dtype": "bf16", "B": 32, "Hq": 12, "Hk": 12, "d": 64, "pos": 40, "n": 200,
         "ragged": True, "H": 16, "W": 16, "rope": "2d", "halves": False},
        # Whole prompts on the high-resolution grid.
        {"name": "append_highres", "op": "append", "dtype": "bf16", "B": 4, "Hq": 24, "Hk": 24, "d": 64, "pos": 0, "n": 4096,
         "ragged": False, "H": 64, "W": 64, "rope": "2d", "halves": False},
        # fp32 storage (checks of a model), shared key heads, rows of odd lengths.
        {"name": "append_f32_ragged", "op": "append", "dtype": "f32", "B": 5, "Hq": 20, "Hk": 4, "d": 64, "pos": 101, "n": 311,
         "ragged": True, "H": 24, "W": 23, "rope": "1d", "halves": True},
        # Prompts of different lengths of the base model, packed.
        {"name": "attend_base_packed", "op": "attend", "dtype": "bf16", "B": 8, "Hq": 12, "Hk": 12, "d": 64, "pos": 0, "n": 256,
         "ragged": True, "window": 128, "sinks": 1},
        # Whole prompts on the high-resolution grid, 16 rows of it back, shared key heads.
        {"name": "attend_highres", "op": "attend", "dtype": "bf16", "B": 4, "Hq": 24, "Hk": 8, "d": 64, "pos": 0, "n": 4096,
         "ragged": False, "window": 1024, "sinks": 16},
        # A few tokens more for two long rows: few queries, many keys.
        {"name": "attend_long_few", "op": "attend", "dtype": "bf16", "B": 2, "Hq": 16, "Hk": 16, "d": 64, "pos": 16000, "n": 24,
         "ragged": True, "window": 16384, "sinks": 64},
        # fp32 storage, shared key heads, a continued batch of odd lengths.
        {"name": "attend_f32_ragged", "op": "attend", "dtype": "f32", "B": 3, "Hq": 20, "Hk": 4, "d": 64, "pos": 101, "n": 311,
         "ragged": True, "window": 96, "sinks": 0},
        # One image sampled by the 12-head model, half a grid back and the class token.  Launch and host latency.
        {"name": "step_one_image", "op": "step", "dtype": "bf16", "B": 1, "Hq": 12, "Hk": 12, "d": 64, "pos": 200, "ragged": False,
         "H": 16, "W": 16, "rope": "2d", "halves": False, "window": 128, "sinks": 1},
        # A serving batch on the high-resolution grid: 16 rows of the grid back, rows of the batch anywhere, shared keys.
        {"name": "step_batch", "op": "step", "dtype": "bf16", "B": 64, "Hq": 24, "Hk": 8, "d": 64, "pos": 2731, "ragged": True,
         "H": 64, "W": 64, "rope": "2d", "halves": False, "window": 1024, "sinks": 16},
        # Two long rows: few heads, many keys each.
        {"name": "step_long", "op": "step", "dtype": "bf16", "B": 2, "Hq": 16, "Hk": 16, "d": 64, "pos": 40000, "ragged": True,
         "H": 256, "W": 256, "rope": "2d", "halves": False, "window": 16384, "sinks": 64},
        # A large batch of long rows that see all of their keys: the cache's bytes.
        {"name": "step_large", "op": "step", "dtype": "bf16", "B": 128, "Hq": 20, "Hk": 20, "d": 64, "pos": 4000, "ragged": True,
         "H": 64, "W": 64, "rope": "2d", "halves": False, "window": 4096, "sinks": 0},
    ]


MOST_SCORES = 4 * 24 * 4096 * 4096         # all query-key pairs, seen or not (the plain form forms them)
MOST_KEYS = 2 ** 30                        # elements of all rows' keys, seen or not


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw(rng):
    op = rng.choice(("append", "attend", "step"))
    Hq = rng.choice((12, 16, 20, 24))
    c = {"op": op, "dtype": "f32" if rng.random() < 0.25 else "bf16", "B": _log_int(rng, 1, 128), "Hq": Hq,
         "Hk": Hq // rng.choice((1, 1, 2, 4)), "d": rng.choice((32, 64, 64, 64, 128)), "ragged": rng.random() < 0.6}
    if op == "step":
        c["pos"] = _log_int(rng, 1, 65535)
    else:
        c["pos"] = _log_int(rng, 1, 16384) if rng.random() < 0.5 else 0
        c["n"] = _log_int(rng, 1, 4096)
    if op != "attend":
        W = rng.randint(8, 256)
        c.update(H=(c["pos"] + c.get("n", 1)) // W + 1, W=W, rope=rng.choice(("2d", "2d", "1d", "none")), halves=rng.random() < 0.4)
    if op != "append":
        c.update(window=_log_int(rng, 16, 16384), sinks=rng.choice((0, 1, 4, 16, 64)))
    return c


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        for k in w:
            largest[c["op"], k] = max(largest.get((c["op"], k), 0), w[k])
    while True:
        c = _draw(rng)
        w = work(c)
        if any(w[k] > largest[c["op"], k] for k in w):
            continue
        keys = c["B"] * (c["pos"] + c.get("n", 1))
        if c["op"] == "append" or (keys * c["Hq"] * c.get("n", 1) <= MOST_SCORES and keys * c["Hk"] * c["d"] <= MOST_KEYS):
            return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(case):
    """Position of the first new token and number of new tokens of every row."""
    p, n = case["pos"], case.get("n", 1)
    if not case["ragged"]:
        return [(p, n)] * case["B"]
    if n == 1:
        return [((p - 41 * b) % (p + 1), 1) for b in range(case["B"])]
    return [((p - 29 * b) % (p + 1), n - b * (n // 2 + 3) % (n + 1)) for b in range(case["B"])]


def _held(case, p, n):
    """Pages of a row that a call reads or writes, by their number in the row."""
    if n == 0:
        return []
    if case["op"] == "append":
        return list(range(p // PAGE, (p + n - 1) // PAGE + 1))
    near = max(0, p - case["window"] + 1) // PAGE
    return list(range(min(near, -(-case["sinks"] // PAGE)))) + list(range(near, (p + n - 1) // PAGE + 1))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, Hq, Hk, d = _type(case), case["B"], case["Hq"], case["Hk"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # the pages of the pool in no order, those that have left the window given back (-1)
    rows = _rows(case)
    held = [_held(case, p, n) for p, n in rows]
    count = sum(len(h) for h in held)
    order = torch.randperm(count, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((B, max(p + n + PAGE - 1 for p, n in rows) // PAGE), -1, dtype=torch.int32)
    filled, at = [0] * count, 0
    for b, (p, n) in enumerate(rows):
        for j in held[b]:
            table[b, j] = order[at]
            filled[order[at]] = max(0, min(PAGE, p + (n if case["op"] == "attend" else 0) - j * PAGE))
            at += 1
    valid = torch.arange(PAGE, device="cuda") < torch.tensor(filled, device="cuda")[:, None]

    def pool(width):
        x = normal(count, Hk, PAGE, width) * valid[:, None, :, None]
        scale = x.abs().amax((2, 3)) / TOP
        return (x / scale.clamp(min=LEAST)[:, :, None, None]).to(torch.float8_e4m3fn), scale

    (kp, ks), (vp, vs) = pool(d), pool(d)
    s = {"case": case, "table": table.cuda(), "pages": (kp, _to_v(vp.view(torch.uint8)).view(torch.float8_e4m3fn), ks, vs),
         "pos": torch.tensor([p for p, _ in rows], dtype=torch.int32, device="cuda")}
    T = sum(n for _, n in rows)
    if case.get("n", 1) > 1:
        s["starts"] = torch.tensor([0] + [n for _, n in rows]).cumsum(0).int().cuda()
    if case["op"] == "attend":
        s["q"] = normal(T, Hq, d).to(dt)                       # (normalised already: unit variance)
        return s
    # (the projection gives q, k and v side by side: they are views of it)
    proj = normal(T, Hq + 2 * Hk, d).to(dt)
    s["q"], s["k"], s["v"] = proj.split((Hq, Hk, Hk), 1)
    if case["op"] == "step":
        s["q"], s["k"], s["v"] = (s[x].contiguous() for x in "qkv")
    s["wq"], s["wk"] = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)
    return s


def _to_v(x):
    """[.., 64 positions, d] in the order of a page of v, [.., d, 64]."""
    return x.unflatten(-2, (4, 4, 4)).movedim(-1, -4).transpose(-3, -2).contiguous().flatten(-3)


def _from_v(x):
    return x.unflatten(-1, (4, 4, 4)).transpose(-3, -2).movedim(-4, -1).contiguous().flatten(-4, -2)


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2507_01652_amd import binding as lasad
    c = s["case"]
    kw = {}
    if c["op"] != "attend":
        kw = dict(q_weight=s["wq"], k_weight=s["wk"], norm_eps=EPS, rope_base=BASE,
                  rope={"none": lasad.ROPE_NONE, "1d": lasad.ROPE_1D, "2d": lasad.ROPE_2D}[c["rope"]],
                  pairing=lasad.PAIR_HALVES if c["halves"] else lasad.PAIR_ADJACENT)
    if c["op"] == "append":
        q = lasad.lasad_append_pages(s["q"], s["k"], s["v"], s["pages"], s["table"], s["pos"], c["H"], c["W"],
                                     row_starts=s.get("starts"), **kw)
        return (q, *s["pages"])
    if c["op"] == "attend":
        return lasad.lasad_forward_pages(s["q"], s["pages"], s["table"], s["pos"], c["window"], c["sinks"], row_starts=s.get("starts"))
    o = lasad.lasad_decode_step_pages(s["q"], s["k"], s["v"], s["pages"], s["table"], s["pos"], c["H"], c["W"], c["window"], c["sinks"], **kw)
    return (o, *s["pages"])


# ---- plain forms --------------------------------------------------------------------------------------------------

def _tokens(s):
    """Row and position of every new token."""
    T, B = s["q"].shape[0], s["case"]["B"]
    if "starts" not in s:
        return torch.arange(B, device="cuda"), s["pos"].long()
    at = torch.arange(T, device="cuda")
    row = torch.searchsorted(s["starts"].long(), at, right=True) - 1
    return row, s["pos"].long()[row] + at - s["starts"].long()[row]


def _rotate(c, x, positions):
    """The pairs of [T, heads, d] turned by their positions: angles in 64 bits."""
    if c["rope"] == "none":
        return x
    half = c["d"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    p = positions.double()[:, None]
    if c["rope"] == "2d":                    # the first half of the pairs turns with the row, the second with the column
        quarter = half // 2
        axis = torch.where(i < quarter, torch.div(p, c["W"], rounding_mode="floor"), p % c["W"])
        angle = axis * BASE ** (-(i % quarter) / quarter)
    else:
        angle = p * BASE ** (-i / half)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if not c["halves"]:
        a, b = x[..., 0::2], x[..., 1::2]
    elif c["rope"] == "2d":
        a, b = (t.flatten(-2) for t in x.unflatten(-1, (2, 2, half // 2)).unbind(-2))
    else:
        a, b = x.chunk(2, dim=-1)
    a, b = a * cos - b * sin, a * sin + b * cos
    if not c["halves"]:
        return torch.stack((a, b), -1).flatten(-2)
    if c["rope"] == "2d":
        return torch.stack((a.unflatten(-1, (2, half // 2)), b.unflatten(-1, (2, half // 2))), -2).flatten(-3)
    return torch.cat((a, b), -1)


def _heads(c, x, w, positions):
    x = x.float()
    return _rotate(c, x * (x * x).mean(-1, keepdim=True).add(EPS).rsqrt() * w, positions)


def _put(s, x, codes, scales, row, positions):
    """x [T, Hk, d] into the pages `codes` [pages, Hk, 64, d] (bytes, a copy) and their scales (in place); the pages again."""
    c = s["case"]
    table, first = s["table"].long(), s["pos"].long()
    page, slot = table[row, positions // PAGE], positions % PAGE
    # tokens that were there before: in the page of a row's first new token
    begun = table.gather(1, (first // PAGE).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    new = (s["starts"].diff() if "starts" in s else torch.ones_like(s["pos"])) > 0
    begun, earlier = begun[new], (first % PAGE)[new]
    old = torch.zeros_like(scales)
    old[begun] = scales[begun] * (earlier > 0)[:, None]
    need = torch.zeros_like(scales).scatter_reduce(0, page[:, None].expand(-1, c["Hk"]), x.abs().amax(-1), "amax")
    ratio, exponent = torch.frexp(need / (TOP * torch.where(old > 0, old, 1.0)))
    grow = torch.ldexp(torch.ones_like(old), (exponent - (ratio == 0.5).int()).clamp(min=0))
    fresh = torch.where(need > 0, (need / TOP).clamp(min=LEAST), 0.0)
    made = torch.where(old > 0, old * grow, fresh)
    touched = torch.zeros(len(scales), dtype=torch.bool, device="cuda")
    touched[page] = True
    scales.copy_(torch.where(touched[:, None], made, scales))
    # earlier codes in steps of the new scale
    was = codes[begun]
    smaller = (was.view(torch.float8_e4m3fn).float() / grow[begun][:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    keep = (torch.arange(PAGE, device="cuda") < earlier[:, None])[:, None, :, None]
    codes[begun] = torch.where(keep, smaller, was)
    scaled = x / torch.where(made > 0, made, 1.0)[page][..., None]
    codes[page, :, slot] = scaled.clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes


def _append(s):
    """The rotated queries in 32 bits; the pages are written."""
    c = s["case"]
    row, positions = _tokens(s)
    kp, vp, ks, vs = s["pages"]
    k = _heads(c, s["k"], s["wk"], positions)
    kb, vb = kp.view(torch.uint8), vp.view(torch.uint8)
    kb.copy_(_put(s, k, kb.clone(), ks, row, positions))
    vb.copy_(_to_v(_put(s, s["v"].float(), _from_v(vb), vs, row, positions)))
    return _heads(c, s["q"], s["wq"], positions)


def _attend(s, q):
    """q [T, Hq, d] in 32 bits over the pages."""
    c = s["case"]
    B, Hq, Hk, d, window, sinks = (c[x] for x in ("B", "Hq", "Hk", "d", "window", "sinks"))
    G = Hq // Hk
    row, positions = _tokens(s)
    kp, vp, ks, vs = s["pages"]
    table = s["table"].long()
    there = table.clamp(min=0)
    m = table.shape[1] * PAGE
    v = _from_v(vp.view(torch.uint8)).view(torch.float8_e4m3fn)
    # the rows' keys one behind the other, queries padded to the longest row
    k, v = ((codes.view(torch.uint8)[there].view(torch.float8_e4m3fn).float() * scale[there][..., None, None]).transpose(1, 2)
            .reshape(B, Hk, m, d) for codes, scale in ((kp, ks), (v, vs)))
    n = c.get("n", 1)
    i = positions - s["pos"].long()[row]
    padded = torch.zeros(B, n, Hq, d, device="cuda")
    padded[row, i] = q
    padded = padded.view(B, n, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, d)
    x = torch.matmul(padded, k.transpose(2, 3).contiguous()).view(B, Hq, n, m) * d ** -0.5
    p = (s["pos"].long()[:, None] + torch.arange(n, device="cuda"))[:, None, :, None]
    j = torch.arange(m, device="cuda")
    seen = (j <= p) & ((p - j < window) | (j < sinks))
    x = x.masked_fill_(~seen, -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp()
    o = torch.matmul(x.view(B, Hk, G * n, m), v).view(B, Hq, n, d) / x.sum(-1, keepdim=True)
    return o.transpose(1, 2)[row, i].to(_type(c))


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "attend":
        return _attend(state, state["q"].float())
    q = _append(state)
    if c["op"] == "append":
        return (q.to(_type(c)), *state["pages"])
    return (_attend(state, q), *state["pages"])


def work(case):
    """Bytes: each input read and each output written once, of the cache the codes that are seen or written (not those of a page
    that is only rescaled).  Operations: the norm's and the rotation's 9 an element; two products over the pairs that are seen."""
    e = 2 if case["dtype"] == "bf16" else 4
    Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
    rows = _rows(case)
    T = sum(n for _, n in rows)
    nbytes, flops = 2 * T * Hq * d * e, 0
    if case["op"] != "attend":
        nbytes += T * Hk * d * 2 * (e + 1)
        flops += T * (Hq + Hk) * d * 9
    if case["op"] != "append":
        window, sinks = case["window"], case["sinks"]
        for p, n in rows:
            if n:
                near = max(0, p - window + 1)
                nbytes += 2 * Hk * d * (p + n - near + min(sinks, near))
                far = sum(min(q + 1, window) + max(0, min(sinks, q - window + 1)) for q in range(p, p + n))
                flops += 4 * d * Hq * far
    return {"bytes": nbytes, "flops": flops}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _turned(c, x, weight, p):
    """[heads, d] of the token at position p: norm, weight, rotation."""
    d = c["d"]
    x = x.double()
    x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + EPS) * weight.double()
    if c["rope"] == "none":
        return x
    span = d // 2 if c["rope"] == "2d" else d                       # channels that one axis turns
    k = torch.arange(span // 2, dtype=torch.float64, device="cuda")
    axes = [p // c["W"], p % c["W"]] if c["rope"] == "2d" else [p]
    angle = torch.cat([a.double()[:, None] / BASE ** (2 * k / span) for a in axes], -1)[:, None]
    turn = torch.polar(torch.ones_like(angle), angle)
    channel = torch.arange(d, device="cuda")
    if c["halves"]:
        lo = channel[channel % span < span // 2]
        hi = lo + span // 2
    else:
        lo, hi = channel[0::2], channel[1::2]
    z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * turn
    y = torch.empty_like(x)
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def _e4m3(x):
    """Rounded to the nearest e4m3 value, ties to even mantissas."""
    _, exponent = torch.frexp(x)
    step = torch.exp2((exponent - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-TOP, TOP)


def _exact_pages(s, x, codes, scales):
    """x: the new tokens in 64 bits; codes in the order of positions.  Row by row, page by page."""
    c = s["case"]
    codes, scales, at = codes.double(), scales.double(), 0
    table = s["table"].tolist()
    for b, (p, n) in enumerate(_rows(c)):
        while n > 0:
            page, first = table[b][p // PAGE], p % PAGE
            some = min(n, PAGE - first)
            new = x[at:at + some].transpose(0, 1)
            most = new.abs().amax((1, 2))
            old = scales[page] if first else torch.zeros_like(most)
            power = torch.ceil(torch.log2((most / (TOP * old)).clamp(min=1.0)))      # (nan and inf where old = 0)
            scales[page] = torch.where(old > 0, old * torch.exp2(power), (most / TOP).clamp(min=LEAST) * (most > 0))
            if first:
                by = torch.where(old > 0, torch.exp2(power), 1.0)
                codes[page, :, :first] = _e4m3(codes[page, :, :first] / by[:, None, None])
            divisor = torch.where(scales[page] > 0, scales[page], 1.0)
            codes[page, :, first:first + some] = _e4m3(new / divisor[:, None, None])
            at, p, n = at + some, p + some, n - some
    return codes, scales


def _exact_attend(s, q, k, v, ks, vs):
    """q [T, Hq, d]; k, v: codes [pages, Hk, 64, d] in the order of positions."""
    c = s["case"]
    G, o, at = c["Hq"] // c["Hk"], torch.zeros_like(q), 0
    table = s["table"].long()
    for b, (p, n) in enumerate(_rows(c)):
        if n == 0:
            continue
        used = torch.tensor(_held(c, p, n), device="cuda")
        j = (used[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
        page = table[b, used]
        for h in range(c["Hk"]):
            kk, vv = ((x[page, h] * sc[page, h, None, None].double()).flatten(0, 1) for x, sc in ((k, ks), (v, vs)))
            for i in range(0, n, 1024):
                i1 = min(n, i + 1024)
                back = torch.arange(p + i, p + i1, device="cuda")[:, None] - j[None]
                hidden = (back < 0) | ((back >= c["window"]) & (j >= c["sinks"])[None])
                x = q[at + i:at + i1, h * G:(h + 1) * G].transpose(0, 1) @ kk.T / math.sqrt(c["d"])
                o[at + i:at + i1, h * G:(h + 1) * G] = (torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ vv).transpose(0, 1)
        at += n
    return o


def exact(case, seed):
    launches = 60e-6 * sum(len(_held(case, p, n)) for p, n in _rows(case)) * 12 if case["op"] == "append" else \
        500e-6 * case["B"] * case["Hk"] * (case.get("n", 1) // 1024 + 1)
    if launches > 15:
        return None
    s = prepare(case, seed)
    kp, vp, ks, vs = s["pages"]
    v = _from_v(vp.view(torch.uint8)).view(torch.float8_e4m3fn)
    if case["op"] == "attend":
        return _exact_attend(s, s["q"].double(), kp.double(), v.double(), ks, vs)
    p = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in _rows(case)])
    q = _turned(case, s["q"], s["wq"], p)
    k, ks = _exact_pages(s, _turned(case, s["k"], s["wk"], p), kp, ks)
    v, vs = _exact_pages(s, s["v"].double(), v, vs)
    if case["op"] == "step":
        q = _exact_attend(s, q, k, v, ks, vs)
    return q, k, _to_v(v), ks, vs
