"""Timed cases of the head norms with raster rotation and of the window attention, in plain torch and through the
framework's calls.

Two operators that a model with some softmax layers between its linear-attention layers runs one after the other:

  qk      every query and key head: root-mean-square norm over its d channels, weight, rotation by the token's raster
          position (or by its row and column).  Kinds "forward", "backward" (gradients of the inputs and of both norm
          weights) and "step" (one token for every batch row).
  window  softmax attention in which position p sees the positions p - window + 1 .. p and the first `sinks`
          positions.  Kinds "forward", "train" (forward, then the gradients of q, k and v) and "step" (one token
          against a cache of sinks + window rows or more, this token's key and value appended).

A case is a dict of plain values:

  op, kind      as above;  dtype  storage type of the token tensors ("bf16", "f32")
  B, Hq, Hk, d  batch rows, query heads, key heads (each shared by Hq / Hk query heads), channels of a head
  H, W          token grid (qk);  start  position of the first token;  n  tokens
  rope, halves  "2d", "1d" or "none"; pairs (i, i + half) instead of (2i, 2i + 1);  shared  one norm weight for all heads
  window, sinks;  m  keys, those of positions 0 .. m - 1;  ragged  a number of valid keys of its own for each batch row
  pos, rows     step: position of batch row 0, and whether the other rows are elsewhere;  cap  rows of the cache
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # One image sampled by the 12-head model: norm and rotation of one token's heads.  Launch and host latency.
        {"name": "qk_step_one_image", "op": "qk", "kind": "step", "dtype": "bf16", "B": 1, "Hq": 12, "Hk": 12, "d": 64,
         "H": 16, "W": 16, "pos": 100, "rows": False, "rope": "2d", "halves": False, "shared": True},
        # The high-resolution grid's teacher-forced pass: every token's heads once through memory.
        {"name": "qk_forward_highres", "op": "qk", "kind": "forward", "dtype": "bf16", "B": 4, "Hq": 24, "Hk": 24, "d": 64,
         "H": 64, "W": 64, "start": 0, "n": 4096, "rope": "2d", "halves": False, "shared": True},
        # Training the 16-head model at 384 pixels: gradients of the projections and of the norm weights, one per head.
        {"name": "qk_backward_large", "op": "qk", "kind": "backward", "dtype": "bf16", "B": 32, "Hq": 16, "Hk": 16, "d": 64,
         "H": 24, "W": 24, "start": 0, "n": 576, "rope": "2d", "halves": False, "shared": False},
        # fp32 storage (checks of a model), shared key heads, an image continued in mid-row, an odd number of tokens.
        {"name": "qk_forward_f32_ragged", "op": "qk", "kind": "forward", "dtype": "f32", "B": 3, "Hq": 20, "Hk": 4, "d": 64,
         "H": 24, "W": 23, "start": 101, "n": 311, "rope": "1d", "halves": True, "shared": True},
        # One image sampled by the 12-head model: half a grid back and the class token.  Launch and host latency.
        {"name": "window_step_one_image", "op": "window", "kind": "step", "dtype": "bf16", "B": 1, "Hq": 12, "Hk": 12, "d": 64,
         "window": 128, "sinks": 1, "pos": 200, "rows": False, "cap": 257},
        # A serving batch on the high-resolution grid: 16 rows of the grid back, rows of the batch anywhere, shared keys,
        # a cache that holds no more than is seen and goes round.
        {"name": "window_step_batch", "op": "window", "kind": "step", "dtype": "bf16", "B": 64, "Hq": 24, "Hk": 8, "d": 64,
         "window": 1024, "sinks": 16, "pos": 2731, "rows": True, "cap": 1040},
        # Two long sequences: few heads, many rows each.
        {"name": "window_step_long", "op": "window", "kind": "step", "dtype": "bf16", "B": 2, "Hq": 16, "Hk": 16, "d": 64,
         "window": 16384, "sinks": 64, "pos": 40000, "rows": True, "cap": 16448},
        # Teacher-forced pass of the base model, 256-pixel images, half a grid back.
        {"name": "window_forward_base", "op": "window", "kind": "forward", "dtype": "bf16", "B": 8, "Hq": 12, "Hk": 12, "d": 64,
         "window": 128, "sinks": 1, "start": 0, "n": 256, "m": 256, "ragged": False},
        # The high-resolution grid, 16 rows of it back.
        {"name": "window_forward_highres", "op": "window", "kind": "forward", "dtype": "bf16", "B": 4, "Hq": 24, "Hk": 24, "d": 64,
         "window": 1024, "sinks": 16, "start": 0, "n": 4096, "m": 4096, "ragged": False},
        # fp32 storage, shared keys, a continued sequence whose batch rows end at different keys: some queries see none.
        {"name": "window_forward_f32_ragged", "op": "window", "kind": "forward", "dtype": "f32", "B": 3, "Hq": 20, "Hk": 4, "d": 64,
         "window": 96, "sinks": 0, "start": 101, "n": 311, "m": 412, "ragged": True},
        # Training the 16-head model at 384 pixels, six rows of the grid back.
        {"name": "window_train_large", "op": "window", "kind": "train", "dtype": "bf16", "B": 32, "Hq": 16, "Hk": 16, "d": 64,
         "window": 144, "sinks": 1, "start": 0, "n": 576, "m": 576, "ragged": False},
        # Training on the high-resolution grid with shared key heads: their gradients are sums over three query heads.
        {"name": "window_train_highres", "op": "window", "kind": "train", "dtype": "bf16", "B": 2, "Hq": 24, "Hk": 8, "d": 64,
         "window": 1024, "sinks": 16, "start": 0, "n": 4096, "m": 4096, "ragged": False},
    ]


MOST_ELEMENTS = 4 * 4096 * 48 * 64         # of q and k together, in a drawn qk case
MOST_CACHE = 2 * 16 * 16448 * 64           # elements of one cache
MOST_SCORES = 2 * 24 * 4096 * 4096         # all query-key pairs, seen or not (the plain form forms them)


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw(rng):
    op = rng.choice(("qk", "window"))
    Hq = rng.choice((12, 16, 20, 24))
    Hk = Hq // rng.choice((1, 1, 2, 4))
    c = {"op": op, "dtype": "f32" if rng.random() < 0.25 else "bf16", "Hq": Hq, "Hk": Hk, "d": rng.choice((32, 64, 64, 64, 128))}
    if op == "qk":
        c.update(kind=rng.choice(("forward", "backward", "step")), H=rng.randint(8, 64), W=rng.randint(8, 64),
                 rope=rng.choice(("2d", "2d", "1d", "none")), halves=rng.random() < 0.4, shared=rng.random() < 0.6)
        if c["kind"] == "step":
            c.update(B=_log_int(rng, 1, 256), pos=rng.randrange(c["H"] * c["W"]), rows=rng.random() < 0.5)
        else:
            start = rng.randrange(c["H"] * c["W"] // 2) if rng.random() < 0.4 else 0
            c.update(B=_log_int(rng, 1, 64), start=start, n=_log_int(rng, 1, c["H"] * c["W"] - start))
        return c
    c.update(kind=rng.choice(("forward", "train", "step")), sinks=rng.choice((0, 1, 4, 16, 64)))
    if c["kind"] == "step":
        c.update(B=_log_int(rng, 1, 256), window=_log_int(rng, 16, 16384), rows=rng.random() < 0.7)
        c["cap"] = c["sinks"] + c["window"] + rng.choice((0, 0, rng.randint(1, 512)))
        c["pos"] = _log_int(rng, 1, 65536)
    else:
        start = _log_int(rng, 1, 4096) if rng.random() < 0.4 else 0
        n = _log_int(rng, 1, 16384)
        c.update(B=_log_int(rng, 1, 64), start=start, n=n, m=start + n, window=_log_int(rng, 16, 4096), ragged=rng.random() < 0.3)
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
        if c["op"] == "qk":
            if c["B"] * c.get("n", 1) * (c["Hq"] + c["Hk"]) * c["d"] <= MOST_ELEMENTS:
                return c
        elif c["kind"] == "step":
            if c["B"] * c["Hk"] * c["cap"] * c["d"] <= MOST_CACHE:
                return c
        elif c["B"] * c["Hq"] * c["n"] * c["m"] <= MOST_SCORES:
            return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _positions(case):
    """Of a step's batch rows."""
    last = case["H"] * case["W"] if case["op"] == "qk" else case["pos"] + 1
    return [(case["pos"] - 41 * b) % last if case["rows"] else case["pos"] for b in range(case["B"])]


def _lengths(case):
    """Valid keys of the batch rows."""
    m = case["m"]
    return [m - (b * (m // 2 + 37)) % (m + 1) for b in range(case["B"])] if case["ragged"] else [m] * case["B"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, Hq, Hk, d = _type(case), case["B"], case["Hq"], case["Hk"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": case}
    step = case["kind"] == "step"
    tokens = (B,) if step else (B, case["n"])
    if case["op"] == "qk":
        # (the projection gives q, k and v side by side: q and k are views of it)
        proj = normal(*tokens, Hq + 2 * Hk, d).to(dt)
        s["q"], s["k"] = proj[..., :Hq, :], proj[..., Hq:Hq + Hk, :]
        if step:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["wq"] = 1 + 0.1 * (normal(d) if case["shared"] else normal(Hq, d))
        s["wk"] = 1 + 0.1 * (normal(d) if case["shared"] else normal(Hk, d))
        if case["kind"] == "backward":
            s["dq"], s["dk"] = normal(*tokens, Hq, d).to(dt), normal(*tokens, Hk, d).to(dt)
    else:
        # (queries and keys have been normalised: unit variance)
        s["q"] = normal(*tokens, Hq, d).to(dt)
        keys = (B,) if step else (B, case["m"])
        s["k"], s["v"] = normal(*keys, Hk, d).to(dt), normal(*keys, Hk, d).to(dt)
        if case["kind"] == "train":
            s["do"] = normal(*tokens, Hq, d).to(dt)
        if step:
            s["kc"] = normal(B, Hk, case["cap"], d).to(dt)
            s["vc"] = normal(B, Hk, case["cap"], d).to(dt)
        elif case["ragged"]:
            s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if step:
        s["pos"] = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
    return s


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2507_01652_amd import binding as lasad
    c = s["case"]
    if c["op"] == "qk":
        kw = dict(q_weight=s["wq"], k_weight=s["wk"], norm_eps=EPS, rope_base=BASE,
                  rope={"none": lasad.ROPE_NONE, "1d": lasad.ROPE_1D, "2d": lasad.ROPE_2D}[c["rope"]],
                  pairing=lasad.PAIR_HALVES if c["halves"] else lasad.PAIR_ADJACENT)
        if c["kind"] == "step":
            return lasad.lasad_decode_step_qk(s["q"], s["k"], c["H"], c["W"], s["pos"] if c["rows"] else c["pos"], **kw)
        if c["kind"] == "forward":
            return lasad.lasad_forward_qk(s["q"], s["k"], c["H"], c["W"], start_pos=c["start"], **kw)
        return lasad.lasad_backward_qk(s["q"], s["k"], s["dq"], s["dk"], c["H"], c["W"], start_pos=c["start"], **kw)
    if c["kind"] == "step":
        o = lasad.lasad_decode_step_window(s["q"], s["k"], s["v"], s["kc"], s["vc"], s["pos"] if c["rows"] else c["pos"],
                                           c["window"], c["sinks"])
        return o, s["kc"], s["vc"]
    kw = dict(sinks=c["sinks"], start_pos=c["start"], kv_lens=s.get("lens"))
    if c["kind"] == "forward":
        return lasad.lasad_forward_window(s["q"], s["k"], s["v"], c["window"], **kw)
    o, lse = lasad.lasad_forward_window(s["q"], s["k"], s["v"], c["window"], want_lse=True, **kw)
    return (o, *lasad.lasad_backward_window(s["q"], s["k"], s["v"], o, lse, s["do"], c["window"], **kw))


# ---- plain forms --------------------------------------------------------------------------------------------------

def _rotation(c, positions):
    """Cosines and sines [.., d / 2] of the pairs at these positions: angles in 64 bits."""
    half = c["d"] // 2
    i = torch.arange(half, device=positions.device, dtype=torch.float64)
    p = positions.double()[..., None]
    if c["rope"] == "2d":                    # the first half of the pairs turns with the row, the second with the column
        quarter = half // 2
        axis = torch.where(i < quarter, torch.div(p, c["W"], rounding_mode="floor"), p % c["W"])
        angle = axis * BASE ** (-(i % quarter) / quarter)
    else:
        angle = p * BASE ** (-i / half)
    return angle.cos().float(), angle.sin().float()


def _pairs(c, x):
    """The two members of every pair: [.., d] -> two of [.., d / 2]."""
    if not c["halves"]:
        return x[..., 0::2], x[..., 1::2]
    if c["rope"] == "2d":
        a, b, e, f = x.chunk(4, dim=-1)
        return torch.cat((a, e), -1), torch.cat((b, f), -1)
    return x.chunk(2, dim=-1)


def _unpairs(c, a, b):
    if not c["halves"]:
        return torch.stack((a, b), -1).flatten(-2)
    if c["rope"] == "2d":
        (a0, a1), (b0, b1) = a.chunk(2, dim=-1), b.chunk(2, dim=-1)
        return torch.cat((a0, b0, a1, b1), -1)
    return torch.cat((a, b), -1)


def _rotate(c, x, cs):
    if c["rope"] == "none":
        return x
    (a, b), (cos, sin) = _pairs(c, x), cs
    return _unpairs(c, a * cos - b * sin, a * sin + b * cos)


def _plain_qk(s):
    c, dt = s["case"], _type(s["case"])
    positions = s["pos"] if c["kind"] == "step" else c["start"] + torch.arange(c["n"], device="cuda")
    cs = tuple(t[..., None, :] for t in _rotation(c, positions))           # the same for every head
    outs, weights = [], []
    for x, w, g in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x = x.float()
        rstd = (x * x).mean(-1, keepdim=True).add(EPS).rsqrt()
        if g is None:
            outs.append(_rotate(c, x * rstd * w, cs).to(dt))
            continue
        g = _rotate(c, g.float(), (cs[0], -cs[1]))
        xh = x * rstd
        gw = g * w
        outs.append(((gw - xh * (gw * xh).mean(-1, keepdim=True)) * rstd).to(dt))
        weights.append((g * xh).double().sum((0, 1, 2) if c["shared"] else (0, 1)).float())
    return (*outs, *weights)


def _plain_step(s):
    c = s["case"]
    B, Hk, d, sinks, window, cap = c["B"], c["Hk"], c["d"], c["sinks"], c["window"], c["cap"]
    G = c["Hq"] // Hk
    p = s["pos"].long()[:, None]

    def slot(j):
        return torch.where(j < sinks, j, sinks + (j - sinks) % (cap - sinks))

    rows = torch.arange(B, device="cuda")
    s["kc"][rows, :, slot(p[:, 0])] = s["k"]
    s["vc"][rows, :, slot(p[:, 0])] = s["v"]
    first = torch.arange(sinks, device="cuda")[None].expand(B, sinks)
    near = p - window + 1 + torch.arange(window, device="cuda")
    seen = torch.cat((first < (p - window + 1).clamp(min=0), near >= 0), 1)
    where = slot(torch.cat((first, near), 1).clamp(min=0))
    index = where[:, None, :, None].expand(B, Hk, sinks + window, d)
    k, v = s["kc"].gather(2, index).float(), s["vc"].gather(2, index).float()
    x = torch.matmul(s["q"].float().view(B, Hk, G, d), k.transpose(2, 3).contiguous()) * d ** -0.5
    x = torch.where(seen[:, None, None, :], x, -math.inf)
    e = (x - x.amax(-1, keepdim=True)).exp()
    o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
    return o.reshape(B, c["Hq"], d).to(_type(c)), s["kc"], s["vc"]


def _plain_window(s):
    c, dt = s["case"], _type(s["case"])
    B, Hq, Hk, d, n, m = (c[x] for x in ("B", "Hq", "Hk", "d", "n", "m"))
    G, scale = Hq // Hk, d ** -0.5
    p = c["start"] + torch.arange(n, device="cuda")[:, None]
    j = torch.arange(m, device="cuda")[None, :]
    seen = (j <= p) & ((p - j < c["window"]) | (j < c["sinks"]))
    seen = seen[None, None].expand(1, 1, n, m)
    if c["ragged"]:
        seen = seen & (j < s["lens"][:, None, None, None])

    def heads(x):                                                          # [B, n, H, d] -> [B, H, n, d]
        return x.float().transpose(1, 2).contiguous()

    q = heads(s["q"])
    k, v = (heads(s[x]).repeat_interleave(G, 1) for x in ("k", "v"))
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = (x - torch.where(top == -math.inf, 0.0, top)).exp()
    total = x.sum(-1, keepdim=True)
    prob = x / torch.where(total == 0, 1.0, total)
    del x
    o = torch.matmul(prob, v)
    if c["kind"] == "forward":
        return o.transpose(1, 2).contiguous().to(dt)
    do = heads(s["do"])
    dv = torch.matmul(prob.transpose(2, 3).contiguous(), do)
    dx = torch.matmul(do, v.transpose(2, 3).contiguous())
    dx = prob * (dx - (do * o).sum(-1, keepdim=True)) * scale
    dq = torch.matmul(dx, k)
    dk = torch.matmul(dx.transpose(2, 3).contiguous(), q)
    dk, dv = (t.view(B, Hk, G, m, d).sum(2) for t in (dk, dv))             # shared heads: the sum over their queries
    return tuple(t.transpose(1, 2).contiguous().to(dt) for t in (o, dq, dk, dv))


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "qk":
        return _plain_qk(state)
    return _plain_step(state) if c["kind"] == "step" else _plain_window(state)


def _seen_pairs(case):
    """Query-key pairs of one head over the whole batch."""
    total = 0
    for length in _lengths(case):
        for p in range(case["start"], case["start"] + case["n"]):
            last = min(p, length - 1)
            near = max(0, last - max(0, p - case["window"] + 1) + 1)
            total += near + max(0, min(case["sinks"], p - case["window"] + 1, length))
        if not case["ragged"]:
            return total * case["B"]
    return total


def work(case):
    """Bytes: each input read and each output written once, of a cache the rows that are seen.  Operations: the norm's
    and the rotation's 3 and 6 an element (twice that for gradients); two products over the pairs that are seen, five
    more for the gradients."""
    e = 2 if case["dtype"] == "bf16" else 4
    B, Hq, Hk, d = case["B"], case["Hq"], case["Hk"], case["d"]
    if case["op"] == "qk":
        rows = B * case.get("n", 1) * (Hq + Hk)
        passes, grad = (3, 2) if case["kind"] == "backward" else (2, 1)
        weights = 4 * d * (2 if case["shared"] else Hq + Hk)
        return {"bytes": rows * d * e * passes + weights * grad, "flops": rows * d * 9 * grad}
    if case["kind"] == "step":
        seen = sum(min(p + 1, case["window"]) + max(0, min(case["sinks"], p - case["window"] + 1)) for p in _positions(case))
        return {"bytes": e * d * (2 * Hk * (seen + B) + 2 * B * Hq), "flops": 4 * d * Hq * seen}
    qs, ks = B * case["n"] * Hq * d * e, B * case["m"] * Hk * d * e
    pairs = _seen_pairs(case) * Hq * d
    if case["kind"] == "forward":
        return {"bytes": 2 * qs + 2 * ks, "flops": 4 * pairs}
    return {"bytes": 4 * qs + 4 * ks, "flops": 14 * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _turns(c, positions):
    """Unit complex numbers [.., d / 2] by which the pairs are multiplied."""
    out = []
    for i in range(c["d"] // 2):
        if c["rope"] == "none":
            a = torch.zeros_like(positions, dtype=torch.float64)
        elif c["rope"] == "1d":
            a = positions.double() / BASE ** (2 * i / c["d"])
        else:
            row, k = i < c["d"] // 4, i % (c["d"] // 4)
            a = (positions // c["W"] if row else positions % c["W"]).double() / BASE ** (4 * k / c["d"])
        out.append(torch.polar(torch.ones_like(a), a))
    return torch.stack(out, -1)


def _members(c):
    """Channel numbers of the first and second member of each pair."""
    d = c["d"]
    if not c["halves"]:
        return [2 * i for i in range(d // 2)], [2 * i + 1 for i in range(d // 2)]
    span = d // 2 if c["rope"] == "2d" else d                               # halves of what one axis turns
    first = [i for i in range(d) if i % span < span // 2]
    return first, [i + span // 2 for i in first]


def _exact_qk(s):
    c = s["case"]
    positions = s["pos"].long() if c["kind"] == "step" else torch.arange(c["start"], c["start"] + c["n"], device="cuda")
    turn = _turns(c, positions).unsqueeze(-2)
    lo, hi = _members(c)

    def rotate(x, turn):
        z = torch.complex(x[..., lo], x[..., hi]) * turn
        y = torch.empty_like(x)
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    outs, weights = [], []
    for x, w, g in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x, w = x.double(), w.double()
        size = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
        rms = torch.sqrt(size * size / c["d"] + EPS)
        if g is None:
            outs.append(rotate(x / rms * w, turn))
            continue
        g = rotate(g.double(), turn.conj())
        # d/dx of (x / rms) w . g
        along = (g * w * x).sum(-1, keepdim=True)
        outs.append(g * w / rms - x * along / (c["d"] * rms ** 3))
        weights.append((g * x / rms).sum(dim=(0, 1, 2) if c["shared"] else (0, 1)))
    return (*outs, *weights)


def _exact_step(s):
    c = s["case"]
    kc, vc = s["kc"].double(), s["vc"].double()
    o = torch.empty(c["B"], c["Hq"], c["d"], dtype=torch.float64, device="cuda")
    ring = c["cap"] - c["sinks"]
    for b, p in enumerate(_positions(c)):
        at = p if p < c["sinks"] else c["sinks"] + (p - c["sinks"]) % ring
        kc[b, :, at], vc[b, :, at] = s["k"][b].double(), s["v"][b].double()
        lo = max(0, p - c["window"] + 1)
        j = torch.arange(p + 1, device="cuda")
        j = j[(j >= lo) | (j < c["sinks"])]
        j = torch.where(j < c["sinks"], j, (j - c["sinks"]) % ring + c["sinks"])
        for h in range(c["Hk"]):
            g = slice(h * (c["Hq"] // c["Hk"]), (h + 1) * (c["Hq"] // c["Hk"]))
            prob = torch.softmax(s["q"][b, g].double() @ kc[b, h, j].T / math.sqrt(c["d"]), -1)
            o[b, g] = prob @ vc[b, h, j]
    return o, kc, vc


def _exact_window(s):
    c = s["case"]
    B, n, m, Hq, d = (c[x] for x in ("B", "n", "m", "Hq", "d"))
    G = Hq // c["Hk"]
    f64 = dict(dtype=torch.float64, device="cuda")
    o, dq = torch.zeros(B, n, Hq, d, **f64), torch.zeros(B, n, Hq, d, **f64)
    dk, dv = torch.zeros(B, m, c["Hk"], d, **f64), torch.zeros(B, m, c["Hk"], d, **f64)
    some = 1024                                                            # queries at a time
    for b, length in enumerate(_lengths(c)):
        for i0 in range(0, n, some):
            i1 = min(n, i0 + some)
            at = torch.arange(c["start"] + i0, c["start"] + i1, device="cuda")
            keys = torch.arange(min(length, c["start"] + i1), device="cuda")
            back = at[:, None] - keys[None, :]
            hidden = (back < 0) | ((back >= c["window"]) & (keys >= c["sinks"])[None, :])
            for h in range(Hq):
                k, v = s["k"][b, :len(keys), h // G].double(), s["v"][b, :len(keys), h // G].double()
                q = s["q"][b, i0:i1, h].double()
                x = (q @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse = torch.logsumexp(x, -1, keepdim=True)                 # -inf where nothing is seen
                prob = torch.exp(x - lse).masked_fill(hidden, 0.0)
                o[b, i0:i1, h] = prob @ v
                if c["kind"] == "train":
                    do = s["do"][b, i0:i1, h].double()
                    dp = do @ v.T
                    ds = prob * (dp - (prob * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                    dq[b, i0:i1, h] = ds @ k
                    dk[b, :len(keys), h // G] += ds.T @ q
                    dv[b, :len(keys), h // G] += prob.T @ do
    return o if c["kind"] == "forward" else (o, dq, dk, dv)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qk":
        return _exact_qk(s)
    if case["kind"] == "step":
        return _exact_step(s)
    # (about 0.3 ms of launches for each batch row, head and 1024 queries)
    if case["B"] * case["Hq"] * (case["n"] // 1024 + 1) > 40_000:
        return None
    return _exact_window(s)
