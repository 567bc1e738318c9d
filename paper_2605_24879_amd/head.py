"""The output head and its cross entropy as a torch module around libdprc.

``Head`` wraps a bias-free ``nn.Linear`` from hidden states to a vocabulary and gives every token's loss
without storing a logit: the forward call keeps the log-sum-exps, the backward call forms the logits again,
a piece of the vocabulary at a time.  Under a private training step (``dpsgd.DPSGDRC`` with ``head=``) the
backward call also estimates every sample's squared norm of its weight gradient, and the step takes the
clipped sum; otherwise the weight gets its ordinary gradient.
"""

import torch
import torch.nn as nn

from . import dprc as D
from .junction import _recorded, token_rows


class _HeadFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, weight, target, mod):
        loss, lse = D.dprc_head_loss(h, weight, target)
        ctx.save_for_backward(h, weight, target, lse)
        ctx.mod = mod
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        h, weight, target, lse = ctx.saved_tensors
        g = g.contiguous()
        want_h, want_w = ctx.needs_input_grad[:2]
        if ctx.mod.sink is not None:
            return ctx.mod.sink(h, weight, target, lse, g, want_h), None, None, None
        dh, dW = D.dprc_head_backward(h, weight, target, lse, g, hidden_grad=want_h, weight_grad=want_w)
        return dh, dW, None, None


class Head(nn.Module):
    """Per-token losses [B, T] (fp32) of hidden states [B, T, d] against target ids [B, T] (int64): cross entropy over
    the outputs of ``linear``.  A negative target has no loss.  ``linear`` stays the owner of the weight.

    In a captured pass take gradients with torch.autograd.grad: torch ends the process where ``backward`` is captured while
    an eager graph of the same leaves lives."""

    def __init__(self, linear):
        super().__init__()
        if linear.bias is not None:
            raise ValueError("the head covers bias-free linear layers")
        self.linear = linear
        self.sink = None                  # a private step's: takes the backward call, returns dh

    def forward(self, h, target):
        h, target, weight = token_rows(h), target.contiguous(), self.linear.weight
        if not _recorded(h, weight):
            return D.dprc_head_loss(h, weight, target)[0]
        return _HeadFn.apply(h, weight, target, self)
