"""fp64 definitions of the output head's cross entropy and its gradients, of rotary positions, and of
clipping by a joint norm (numpy, no code shared with the library)."""

import numpy as np


def loss(h, W, target):
    """(loss, lse) [B, T] of logits h W^T; a negative target has no loss."""
    logits = h @ W.T
    top = logits.max(-1, keepdims=True)
    lse = (top + np.log(np.exp(logits - top).sum(-1, keepdims=True)))[..., 0]
    picked = np.take_along_axis(logits, np.maximum(target, 0)[..., None], -1)[..., 0]
    return np.where(target < 0, 0.0, lse - picked), lse


def errors(h, W, target, lse, g):
    """E [B, T, V] = g (exp(logit - lse) - onehot(target)), zero rows for negative targets."""
    kept = target >= 0
    p = np.exp(np.where(kept[..., None], h @ W.T - lse[..., None], -np.inf))
    b, t = np.nonzero(kept)
    p[b, t, target[b, t]] -= 1.0
    return p * np.where(kept, g, 0.0)[..., None]


def rotary(x, freqs, pos, scale=1.0, interleaved=False, inverse=False):
    """x [B, T, H, D] with its first 2 len(freqs) features turned by pos [B, T] times freqs."""
    r = len(freqs)
    y = x.copy()
    angle = pos[:, :, None, None].astype(np.float64) * freqs
    cos, sin = scale * np.cos(angle), scale * np.sin(angle) * (-1.0 if inverse else 1.0)
    ia = np.arange(r) * 2 if interleaved else np.arange(r)
    ib = ia + 1 if interleaved else ia + r
    y[..., ia] = x[..., ia] * cos - x[..., ib] * sin
    y[..., ib] = x[..., ib] * cos + x[..., ia] * sin
    return y


def clip(tensors, max_norm):
    """(min(1, max_norm / norm) x for every tensor, norm)."""
    norm = np.sqrt(sum((t * t).sum() for t in tensors))
    c = min(1.0, max_norm / norm) if norm > 0 else 1.0
    return [c * t for t in tensors], norm
