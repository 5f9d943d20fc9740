"""Rotary positions of queries and keys (call 9), before the attention calls.

A Rotary holds the frequencies of one kind of positions on the GPU and turns
queries and keys, or their gradients back, through the C ABI; nothing here
computes on the GPU.  It takes the projections where they lie (any strides of
heads and tokens) and writes the layer's layout [heads][n][d].
"""
from __future__ import annotations

import math

import torch

from . import binding as B
from .layer import _allocating_on, _refuse_tangents


def frequencies(length, theta=10000.0, scaling=None, context=4096):
    """(radians per position of the length / 2 pairs, factor on the turned
    channels).  Pair i turns by theta^(-2 i / length); scaling = (kind, s) adapts
    that to contexts s times as long as `context`:
      linear  every frequency divided by s;
      base    theta times s^(length / (length - 2)), which slows the slowest pair s
              times and leaves the fastest (length > 2);
      ramp    pairs that turn less than once over `context` divided by s, those
              that turn more than 32 times left, between them in proportion to how
              often they turn (not to their index); the turned channels times
              1 + 0.1 ln s."""
    kind, s = scaling or (None, 1.0)
    if kind not in (None, "linear", "base", "ramp"):
        raise ValueError(f"scaling {kind!r}: linear, base or ramp")
    if not (math.isfinite(s) and s > 0 and math.isfinite(theta) and theta > 0):
        raise ValueError("theta and the scaling must be positive and finite")
    if kind == "base":
        if length <= 2:
            raise ValueError("base scaling needs more than one pair")
        theta *= s ** (length / (length - 2))
    f = [theta ** (-2 * i / length) for i in range(length // 2)]
    if kind == "linear":
        return [x / s for x in f], 1.0
    if kind == "ramp":
        kept = [min(max((context * x / (2 * math.pi) - 1) / 31, 0.0), 1.0) for x in f]
        return [x * (m + (1 - m) / s) for x, m in zip(f, kept)], 1.0 + 0.1 * math.log(s)
    return f, 1.0


def grid_positions(grid, device="cuda"):
    """int32 [3][n]: the (t, h, w) places of a latent grid's tokens in raster order."""
    t, h, w = map(int, grid)
    i = torch.arange(t * h * w, dtype=torch.int32, device=device)
    return torch.stack((i // (h * w), i // w % h, i % w))


class _RotaryFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, x2, owner, positions, inverse, stream):
        ctx.save_for_backward(positions)
        ctx.owner, ctx.inverse, ctx.two = owner, inverse, x2 is not None
        out = owner._call(x, positions, x2, None, inverse, stream)
        return out if ctx.two else (out, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_y, d_y2):
        positions, = ctx.saved_tensors
        need = [bool(n) for n in ctx.needs_input_grad[:2]]
        d = [g.contiguous() if n else None for g, n in zip((d_y, d_y2), need)]
        grads = [None, None]
        if need[0] and need[1]:
            grads = list(ctx.owner._call(d[0], positions, d[1], None, not ctx.inverse, None))
        elif any(need):
            i = need.index(True)
            grads[i] = ctx.owner._call(d[i], positions, None, None, not ctx.inverse, None)
        return (*grads, None, None, None, None)


class Rotary:
    """Turns channels by positions along one to three axes: `lengths[a]` channels of
    each head for axis a, from `offsets[a]` on (one after the other from channel 0),
    the rest left as they are.  layout "pairs" turns neighbouring channels (2 i, 2 i
    + 1) of an axis' range together, "halves" (i, i + length / 2)."""

    def __init__(self, d, lengths=None, offsets=None, theta=10000.0, layout="pairs", scaling=None,
                 context=4096, device="cuda"):
        self.d, self.layout = int(d), layout
        lengths = [self.d] if lengths is None else [int(x) for x in lengths]
        if offsets is None:
            offsets = [sum(lengths[:i]) for i in range(len(lengths))]
        self.ranges = (tuple(int(x) for x in offsets), tuple(lengths))
        if layout not in B.LAYOUTS:
            raise ValueError(f"layout {layout!r}: pairs or halves")
        if not 1 <= len(lengths) <= 3 or len(self.ranges[0]) != len(lengths):
            raise ValueError("need 1..3 axes, an offset for each")
        if any(n < 2 or n % 2 for n in lengths):
            raise ValueError("an axis needs an even number of channels")
        turns, self.factor = [], 1.0
        for n in lengths:
            f, self.factor = frequencies(n, theta, scaling, context)
            # units of 2^-64 of a turn, as a signed word
            turns += [round(x / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for x in f]
        turns = [x - 2 ** 64 if x >= 2 ** 63 else x for x in turns]
        self.turns = torch.tensor(turns, dtype=torch.int64, device=device)

    def _call(self, x, positions, x2, out, inverse, stream):
        if out is None:
            with _allocating_on(stream):
                out = [torch.empty(t.shape, dtype=t.dtype, device=t.device)
                       for t in (x, x2) if t is not None]
        y, y2 = out if x2 is not None else (out[0], None)
        B.scope_rotary(x, y, positions, self.turns, self.ranges, self.layout, inverse, self.factor,
                       x2, y2, stream)
        return (y, y2) if x2 is not None else y

    def rotate(self, x, positions, x2=None, out=None, inverse=False, stream=None):
        """x [heads][n][d] (bf16 or fp32, any strides of heads and tokens) turned by
        positions, int32 [axes][n] or, with one axis, [n]; with x2, of other heads,
        both by one launch, as a pair.  inverse turns back, times the same factor:
        the gradient.  Into `out` (a tensor, or a pair with x2; each may be its own
        input, not the other's) or new tensors [heads][n][d].  Differentiable in x and x2 (in
        reverse mode; forward mode is refused) except into `out`, which is refused
        where a gradient is asked for."""
        if x.dim() != 3 or x.shape[2] != self.d:
            raise ValueError(f"x must be [heads][n][{self.d}], is {tuple(x.shape)}")
        if x2 is not None and (x2.dim() != 3 or x2.shape[1:] != x.shape[1:] or x2.dtype != x.dtype):
            raise ValueError(f"x2 is {tuple(x2.shape)} {x2.dtype}, x {tuple(x.shape)} {x.dtype}")
        n, axes = x.shape[1], len(self.ranges[0])
        if positions.shape != (axes, n) and (axes > 1 or positions.shape != (n,)):
            raise ValueError(f"positions must be [{axes}][{n}], is {tuple(positions.shape)}")
        given = () if out is None else tuple(out) if isinstance(out, (tuple, list)) else (out,)
        if out is not None and (len(given) != (1 if x2 is None else 2)
                                or any([t is None for t in given])):
            raise ValueError("out needs a tensor for each input")
        _refuse_tangents("rotate", x, x2, *given)
        if torch.is_grad_enabled() and any([t is not None and t.requires_grad
                                            for t in (x, x2, *given)]):
            if given:
                raise ValueError("rotate into `out` is not differentiable: leave `out` away, or "
                                 "call it under torch.no_grad()")
            with _allocating_on(stream):  # the backward pass runs on this stream too
                y, y2 = _RotaryFunction.apply(x, x2, self, positions, bool(inverse), stream)
            return y if x2 is None else (y, y2)
        return self._call(x, positions, x2, given or None, inverse, stream)
