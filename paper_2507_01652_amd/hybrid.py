"""A small raster model with linear and softmax layers in turn, trained and then sampled token by token.

    python -m paper_2507_01652_amd.hybrid [--steps 60] [--grid 16] [--width 256] [--layers 4] [--fp32]

Every second layer is softmax attention: projections, the norm and rotation of its query and key heads
(`lasad_forward_qk`), attention over the last `window` positions and the class token (`lasad_forward_window`, one sink);
the others are the fused linear layer (`lasad_forward_layer`).  Training runs their backward calls from autograd, sampling
their one-token calls, over a state per linear layer and a cache of sinks + window rows per softmax layer: neither grows with
the image.  The projections and the channel mixing are torch products.  The images are synthetic: every image repeats a
pattern that its class picks, so that a token is known from the class and from the row above.
"""
from __future__ import annotations

import argparse

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

from . import binding as lasad

HEAD = 64                    # channels of a head, the fused linear layer's


class _HeadNorms(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, grid):
        ctx.save_for_backward(q, k, q_weight, k_weight)
        ctx.grid = grid
        return lasad.lasad_forward_qk(q, k, *grid, q_weight, k_weight)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_q, d_k):
        q, k, q_weight, k_weight = ctx.saved_tensors
        return (*lasad.lasad_backward_qk(q, k, d_q, d_k, *ctx.grid, q_weight, k_weight), None)


class _Window(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, sinks):
        o, lse = lasad.lasad_forward_window(q, k, v, window, sinks, want_lse=True)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.window, ctx.sinks = window, sinks
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o):
        return (*lasad.lasad_backward_window(*ctx.saved_tensors, d_o.contiguous(), ctx.window, ctx.sinks), None, None)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q_pre, z, v, weight, grid):
        ctx.save_for_backward(q_pre, z, v, weight)
        ctx.grid = grid
        return lasad.lasad_forward_layer(q_pre, z, v, *grid, norm_weight=weight)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o):
        q_pre, z, v, weight = ctx.saved_tensors
        return (*lasad.lasad_backward_layer(q_pre, z, v, d_o.contiguous(), *ctx.grid, norm_weight=weight), None)


def _count_heads(width: int) -> int:
    if width < HEAD or width % HEAD:
        raise ValueError(f"a width of {width} is not a number of heads of {HEAD} channels")
    return width // HEAD


class SoftmaxLayer(torch.nn.Module):
    """Heads of `width`, a key head for every `group` of them (more, where that does not divide them); sees `window` positions back and
    the first `sinks`."""

    def __init__(self, width: int, grid: tuple, window: int, sinks: int = 1, group: int = 2):
        super().__init__()
        self.grid, self.window, self.sinks = grid, window, sinks
        self.hq = _count_heads(width)
        self.hk = max(h for h in range(1, max(1, self.hq // group) + 1) if self.hq % h == 0)
        self.project = torch.nn.Linear(width, (self.hq + 2 * self.hk) * HEAD, bias=False)
        self.out = torch.nn.Linear(width, width, bias=False)
        self.q_weight = torch.nn.Parameter(torch.ones(HEAD))
        self.k_weight = torch.nn.Parameter(torch.ones(HEAD))

    def _heads(self, x):
        return self.project(x).unflatten(-1, (-1, HEAD)).split((self.hq, self.hk, self.hk), -2)

    def forward(self, x):
        q, k, v = self._heads(x)
        q, k = _HeadNorms.apply(q, k, self.q_weight, self.k_weight, self.grid)
        return self.out(_Window.apply(q, k, v, self.window, self.sinks).flatten(-2))

    def begin(self, B: int, dtype, device):
        return tuple(torch.zeros(B, self.hk, self.sinks + self.window, HEAD, dtype=dtype, device=device) for _ in range(2))

    def step(self, x, caches, pos: int):
        q, k, v = (t.contiguous() for t in self._heads(x))
        q, k = lasad.lasad_decode_step_qk(q, k, *self.grid, pos, self.q_weight, self.k_weight)
        return self.out(lasad.lasad_decode_step_window(q, k, v, *caches, pos, self.window, self.sinks).flatten(-2))


class LinearLayer(torch.nn.Module):
    def __init__(self, width: int, grid: tuple):
        super().__init__()
        self.grid, self.heads = grid, _count_heads(width)
        self.project = torch.nn.Linear(width, 3 * width, bias=False)
        self.out = torch.nn.Linear(width, width, bias=False)
        self.o_weight = torch.nn.Parameter(torch.ones(self.heads, HEAD))

    def _heads(self, x):
        q_pre, z, v = self.project(x).unflatten(-1, (3, self.heads, HEAD)).unbind(-3)
        return q_pre, z + 2, v                         # (gates start open: sigmoid(2) = 0.88)

    def forward(self, x):
        return self.out(_Linear.apply(*(t.contiguous() for t in self._heads(x)), self.o_weight, self.grid).flatten(-2))

    def begin(self, B: int, dtype, device):
        return torch.zeros(B, self.heads, HEAD, HEAD, device=device)

    def step(self, x, state, pos: int):
        q_pre, z, v = (t.contiguous() for t in self._heads(x))
        return self.out(lasad.lasad_decode_step_layer(q_pre, z, v, state, *self.grid, pos, norm_weight=self.o_weight).flatten(-2))


class Model(torch.nn.Module):
    """Logits of the grid's tokens in raster order from the class and the tokens before each."""

    def __init__(self, width: int, layers: int, grid: tuple, vocabulary: int, classes: int, window: int):
        super().__init__()
        self.grid = grid
        self.classes = torch.nn.Embedding(classes, width)
        self.tokens = torch.nn.Embedding(vocabulary, width)
        self.layers = torch.nn.ModuleList(SoftmaxLayer(width, grid, window) if i % 2 else LinearLayer(width, grid) for i in range(layers))
        self.mixers = torch.nn.ModuleList(
            torch.nn.Sequential(torch.nn.Linear(width, 2 * width), torch.nn.SiLU(), torch.nn.Linear(2 * width, width))
            for _ in range(layers))
        self.head = torch.nn.Linear(width, vocabulary)

    def _norm(self, x):
        return F.rms_norm(x, x.shape[-1:])

    def forward(self, classes, tokens):
        x = torch.cat((self.classes(classes)[:, None], self.tokens(tokens[:, :-1])), 1)
        for layer, mixer in zip(self.layers, self.mixers):
            x = x + layer(self._norm(x))
            x = x + mixer(self._norm(x))
        return self.head(self._norm(x))

    @torch.no_grad()
    def sample(self, classes, given=None):
        """Tokens [B, N], the likeliest each, and their logits; with `given` tokens these are fed instead of the sampled ones."""
        x = self.classes(classes)
        dtype = torch.get_autocast_dtype("cuda") if torch.is_autocast_enabled("cuda") else x.dtype
        memory = [layer.begin(x.shape[0], dtype, x.device) for layer in self.layers]
        tokens, logits = [], []
        for pos in range(self.grid[0] * self.grid[1]):
            for layer, mixer, m in zip(self.layers, self.mixers, memory):
                x = x + layer.step(self._norm(x), m, pos)
                x = x + mixer(self._norm(x))
            logits.append(self.head(self._norm(x)))
            tokens.append(logits[-1].argmax(-1))
            x = self.tokens(tokens[-1] if given is None else given[:, pos])
        return torch.stack(tokens, 1), torch.stack(logits, 1)


def images(B: int, grid: tuple, classes: int, vocabulary: int, generator) -> tuple:
    """A class and its image: row r is the class's first row, turned by r times the class's shift."""
    H, W = grid
    label = torch.randint(classes, (B,), generator=generator)
    first = torch.stack([torch.randint(vocabulary, (W,), generator=torch.Generator().manual_seed(c)) for c in range(classes)])[label]
    at = (torch.arange(W)[None, None] + torch.arange(H)[None, :, None] * (1 + label[:, None, None] % 3)) % W
    return label, first[:, None].expand(B, H, W).gather(2, at).reshape(B, H * W)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--grid", type=int, default=16)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--fp32", action="store_true", help="fp32 storage instead of bf16 (parameters are fp32 in both)")
    args = ap.parse_args(argv)
    grid, vocabulary, classes = (args.grid, args.grid), 64, 8
    torch.manual_seed(0)
    model = Model(args.width, args.layers, grid, vocabulary, classes, window=args.grid * args.grid // 2).cuda()
    storage = torch.autocast("cuda", torch.bfloat16, enabled=not args.fp32)
    optimizer = torch.optim.AdamW(model.parameters(), lr=2e-3)
    generator = torch.Generator().manual_seed(1)
    losses = []
    for step in range(args.steps):
        label, tokens = (t.cuda() for t in images(args.batch, grid, classes, vocabulary, generator))
        with storage:
            logits = model(label, tokens)
        loss = F.cross_entropy(logits.float().flatten(0, 1), tokens.flatten())
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
        if step % 10 == 0 or step == args.steps - 1:
            print(f"step {step:4d}  loss {losses[-1]:.4f}", flush=True)
    label, tokens = (t.cuda() for t in images(4, grid, classes, vocabulary, generator))
    with torch.no_grad(), storage:
        whole = model(label, tokens).float()
        _, stepped = model.sample(label, given=tokens)
        sampled, _ = model.sample(label)
    apart = ((stepped.float() - whole).norm() / whole.norm()).item()
    right = (sampled == tokens).float().mean().item()
    print(f"token by token against the whole pass: logits {apart:.2e} apart; sampled tokens right: {right:.3f}", flush=True)
    return losses, apart, right


if __name__ == "__main__":
    main()
