"""Rotary positions as a torch module around libdprc.

``Rotary`` turns the pairs of every head's first ``dim`` features by position * frequency, for q and k in one
call.  Its backward pass is the same call on the gradients, turning back; nothing but the positions is kept
for it.  The frequencies may be scaled for contexts longer than a model was trained on.
"""

import math

import torch
import torch.nn as nn

from . import dprc as D
from .junction import _recorded


def frequencies(dim, base=10000.0, scaling=None):
    """(radians a position of the dim / 2 pairs as fp64 [dim / 2], the factor of cosine and sine).

    base^(-2 j / dim), scaled by ``scaling``, a dict with "kind" and
    "linear":     "factor" s: every frequency divided by s (positions interpolated);
    "ntk":        "factor" s: the base times s^(dim / (dim - 2)), so that the slowest pair is divided by s and the
                  fastest unchanged;
    "wavelength": "factor" s, "low", "high", "original" (context length L): divided by s where the wavelength
                  exceeds L / low, unchanged below L / high, and in between (1 - a) / s + a times the frequency
                  with a = (L / wavelength - low) / (high - low);
    "ramp":       "factor" s, "original" L, "fast" (32) and "slow" (1) turns over L: with j(n) = dim log(L / (2 pi n)) /
                  (2 log base), pairs before floor(j(fast)) are unchanged, those from ceil(j(slow)) on divided by
                  s, linearly between (YaRN, Peng et al.); cosine and sine times "attention" (by default 0.1 log
                  s + 1).
    """
    if dim < 2 or dim % 2:
        raise ValueError("rotary positions turn an even number of features")
    j = torch.arange(dim // 2, dtype=torch.float64)
    freqs = float(base) ** (-2.0 * j / dim)
    if scaling is None:
        return freqs, 1.0
    kind, s = scaling["kind"], float(scaling["factor"])
    if kind == "linear":
        return freqs / s, 1.0
    if kind == "ntk":
        if dim == 2:
            return freqs, 1.0
        return (float(base) * s ** (dim / (dim - 2))) ** (-2.0 * j / dim), 1.0
    L = float(scaling["original"])
    if kind == "wavelength":
        low, high = float(scaling["low"]), float(scaling["high"])
        a = ((L * freqs / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return freqs * ((1.0 - a) / s + a), 1.0
    if kind == "ramp":
        at = lambda turns: dim * math.log(L / (2.0 * math.pi * turns)) / (2.0 * math.log(base))
        first = max(math.floor(at(float(scaling.get("fast", 32.0)))), 0)
        last = min(math.ceil(at(float(scaling.get("slow", 1.0)))), dim - 1)
        a = ((j - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        return freqs * (a / s + 1.0 - a), float(scaling.get("attention", 0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0))
    raise ValueError(f"unknown scaling {kind!r}")


class _RotaryFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, freqs, pos, start, args, heads_first, out_dtype, *xs):
        ctx.save_for_backward(freqs, pos)
        ctx.start, ctx.args, ctx.dtype = start, args, xs[0].dtype
        return tuple(D.dprc_rotary(list(xs), freqs, pos=pos, start=start, heads_first=heads_first, out_dtype=out_dtype, **args))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *gs):
        freqs, pos = ctx.saved_tensors
        gs = [g if g.stride(3) == 1 else g.contiguous() for g in gs]
        back = D.dprc_rotary(gs, freqs, pos=pos, start=ctx.start, out_dtype=ctx.dtype, **dict(ctx.args, inverse=True))
        return None, None, None, None, None, None, *back


class Rotary(nn.Module):
    """Rotary positions of heads of width ``head_dim``: the first ``dim`` features (all by default), pair j at (j,
    dim / 2 + j), or (2 j, 2 j + 1) with ``interleaved``; ``base`` and ``scaling`` as in ``frequencies``.

    ``rotary(q, k)`` turns [B, T, heads, head_dim] tensors (up to four, one type) and returns as many: at positions
    ``pos`` [B, T] (int64), or ``start`` + t.  Results are of ``out_dtype`` (the inputs' by default), in the memory
    order [B, T, heads, head_dim], or [B, heads, T, head_dim] with ``heads_first``.  The first call on a device copies
    the frequencies there, so it has to come before a graph capture."""

    def __init__(self, head_dim, dim=None, base=10000.0, interleaved=False, scaling=None):
        super().__init__()
        dim = head_dim if dim is None else dim
        if dim > head_dim:
            raise ValueError(f"{dim} features of a head of {head_dim}")
        self.head_dim, self.interleaved = head_dim, bool(interleaved)
        # a plain attribute: a buffer would follow the model to bfloat16
        self.freqs, self.scale = frequencies(dim, base, scaling)
        self._on = {}

    def on(self, device):
        """The frequencies on a device."""
        if device not in self._on:
            with torch.inference_mode(False):   # they may be saved for a backward pass later on
                self._on[device] = self.freqs.to(device)
        return self._on[device]

    def forward(self, *xs, pos=None, start=0, heads_first=False, out_dtype=None):
        if any(x.shape[-1] != self.head_dim for x in xs):
            raise ValueError(f"heads must be {self.head_dim} wide")
        xs = [x if x.stride(3) == 1 else x.contiguous() for x in xs]
        freqs, args = self.on(xs[0].device), dict(scale=self.scale, interleaved=self.interleaved)
        if _recorded(*xs):
            out = _RotaryFn.apply(freqs, pos, start, args, heads_first, out_dtype, *xs)
        else:
            out = D.dprc_rotary(xs, freqs, pos=pos, start=start, heads_first=heads_first, out_dtype=out_dtype, **args)
        return out[0] if len(xs) == 1 else tuple(out)
