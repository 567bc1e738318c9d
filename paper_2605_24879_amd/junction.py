"""The junction between two linear layers of a block as a torch module around libdprc.

``Junction`` computes ``s = res + dropout(x)`` and ``y = norm(s)`` in one call and hands both on:
``y`` to the next layer, ``s`` to the next residual sum.  Its backward pass is one call too, and
forms the gradient of the norm's weight and bias for every sample by itself.  Under a private
training step (``dpsgd.DPSGDRC`` with ``norms=``) these per-sample gradients go to the step, which
adds their squared norms to the estimates and takes their clipped sum; otherwise their sum is the
parameters' ordinary gradient.

``Dropout`` is the same dropout on its own, inside a branch or with a residual that no norm follows.

The dropout mask is a function of (seed, site, row, column) and is made again in the backward pass.
Rows are counted from 0 in every call, so calls on parts of a batch need a seed each.
``seed`` is an attribute: every module that runs in a private step takes the step's key, unless its
caller has set another; without a step the caller changes it from one training step to the next.
"""

import contextlib
import threading

import torch
import torch.nn as nn
from torch.autograd import forward_ad

from . import dprc as D

_KINDS = {"layer": D.LAYERNORM, "rms": D.RMSNORM}


_step = threading.local()               # key: that of the private step under way on this thread


@contextlib.contextmanager
def step_key(key):
    """Within: the key of every module's mask, but those whose seed the caller has set."""
    outer, _step.key = getattr(_step, "key", None), key
    try:
        yield
    finally:
        _step.key = outer


class _Keyed(nn.Module):
    """A module with a dropout mask of key ``seed``."""

    _seed, _own = 0, False              # the key; whether the caller has set it

    @property
    def seed(self):
        return self._seed

    @seed.setter
    def seed(self, value):
        self._seed, self._own = value, value != getattr(_step, "key", None)

    def mask_seed(self):
        key = getattr(_step, "key", None)
        if key is not None and not self._own:
            self._seed = key
        return self._seed


def token_rows(x):
    """x [B, T, n] itself where its token rows have one stride, else a contiguous copy.  (The last token of
    every sample, x[:, -1:], is such rows: one token has no stride of its own, and neither has one sample.)"""
    (B, T, n), (s0, s1, s2) = x.shape, x.stride()
    ld = s1 if T > 1 else s0 if B > 1 else n
    return x if s2 == 1 and ld >= n and (B == 1 or s0 == T * ld) else x.contiguous()


def _recorded(*tensors):
    """Whether a call goes through autograd: gradients are on, or a tensor has a forward-mode tangent, which
    autograd refuses and a call past it would drop.  (Outside a dual level, as torch counts them, none has;
    asking each tensor costs 0.3 us.)"""
    return torch.is_grad_enabled() or getattr(forward_ad, "_current_level", 0) >= 0 and any(
        t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


class _JunctionFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, res, weight, bias, mod, p):
        ctx.args = dict(kind=mod.kind, p=p, seed=mod.mask_seed(), site_id=mod.site_id)
        y, s, mean, rstd = D.dprc_layernorm(x, weight, bias, eps=mod.eps, res=res, **ctx.args)
        ctx.save_for_backward(s, weight, mean, rstd)
        ctx.mod, ctx.has_res, ctx.has_bias = mod, res is not None, bias is not None
        ctx.set_materialize_grads(False)
        return (y,) if s is x else (y, s)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, ds=None):
        s, weight, mean, rstd = ctx.saved_tensors
        mod, B = ctx.mod, s.shape[0]
        dy = torch.zeros_like(s) if dy is None else token_rows(dy)
        ds = None if ds is None else token_rows(ds)
        dw = db = gw = gb = None
        want_w, want_b = ctx.needs_input_grad[2], ctx.has_bias and ctx.needs_input_grad[3]
        if mod.sink is not None:
            dw, db = mod.sink(B)
            want_w, want_b = True, ctx.has_bias
        dx, dh, dw, db = D.dprc_layernorm_backward(dy, s, weight, mean, rstd, ds=ds, weight_grad=want_w,
                                                   bias_grad=want_b, dw=dw, db=db, **ctx.args)
        if mod.sink is None and (want_w or want_b):
            ones = torch.ones(B, dtype=torch.float32, device=s.device)
            gw = D.dprc_clip_accumulate_vectors(dw, ones).to(weight.dtype) if want_w else None
            gb = D.dprc_clip_accumulate_vectors(db, ones).to(weight.dtype) if want_b else None
        return dx if dh is None else dh, dx if ctx.has_res else None, gw, gb, None, None


class Junction(_Keyed):
    """Dropout, residual sum and norm of [B, T, n] token rows: ``y, s = junction(x, res)``.

    ``kind``: "layer" (with a bias unless ``bias`` is false) or "rms" (none).  ``p``: dropout rate,
    in training only.  ``site_id``: the place in the model, part of the mask's key.
    """

    def __init__(self, n, kind="layer", eps=1e-5, bias=True, p=0.0, site_id=0):
        super().__init__()
        self.kind, self.eps, self.p, self.site_id = _KINDS[kind], float(eps), float(p), int(site_id)
        self.weight = nn.Parameter(torch.ones(n))
        self.bias = nn.Parameter(torch.zeros(n)) if kind == "layer" and bias else None
        self.sink = None                  # a private step's: B -> (dw, db) rows to write

    def parameters_in_order(self):
        return [self.weight] if self.bias is None else [self.weight, self.bias]

    def forward(self, x, res=None):
        p = self.p if self.training else 0.0
        x = token_rows(x)
        res = None if res is None else token_rows(res)
        if not _recorded(x, res, self.weight, self.bias):
            y, s, _, _ = D.dprc_layernorm(x, self.weight, self.bias, eps=self.eps, kind=self.kind, res=res, p=p,
                                          seed=self.mask_seed(), site_id=self.site_id, stats=False)
            return y, s
        out = _JunctionFn.apply(x, res, self.weight, self.bias, self, p)
        return out if len(out) == 2 else (out[0], x)


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, res, p, seed, site_id):
        ctx.args, ctx.has_res = (p, seed, site_id), res is not None
        return D.dprc_dropout(x, p, seed, site_id, res=res)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = D.dprc_dropout(token_rows(dy), *ctx.args) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.has_res else None, None, None, None


class Dropout(_Keyed):
    """Dropout of [B, T, n] token rows, and the residual added: ``res + dropout(x)`` (x itself where there is
    neither).  Nothing is kept for the backward pass.  ``p``, in training only, ``site_id`` and ``seed`` as in
    ``Junction``."""

    def __init__(self, p, site_id=0):
        super().__init__()
        self.p, self.site_id = float(p), int(site_id)

    def forward(self, x, res=None):
        p = self.p if self.training else 0.0
        if res is None and p == 0.0:
            return x
        x = token_rows(x)
        res = None if res is None else token_rows(res)
        seed = self.mask_seed()
        if not _recorded(x, res):
            return D.dprc_dropout(x, p, seed, self.site_id, res=res)
        return _DropoutFn.apply(x, res, p, seed, self.site_id)
