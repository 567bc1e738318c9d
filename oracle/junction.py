"""fp64 reference of what lies between two linear layers of a block: dropout, residual sum, norm.

TEST INFRASTRUCTURE: see the package docstring.

Everything takes rows [B, T, n] and works in float64 from the definitions.  The dropout mask is
a function of (seed, site, row, column): with row r = i*T + t, the 16 bits of element (r, c) are
half (c mod 2) (0 = low) of word (c mod 8) div 2 of Philox(counter = (c div 8, r, site, 4), key =
(seed mod 2^32, seed div 2^32)); with q = floor(65536 p + 1/2) it is dropped iff they are below q.
p is taken as the binary32 number that the C interface takes.
"""

import numpy as np

from . import philox
from .estimators import as_f64

STREAM_DROPOUT = 4


def dropout_bits(seed, site, rows, n, row0=0):
    """The 16 random bits of every element: uint16 [rows, n]."""
    nb = (n + 7) // 8
    ctr = np.zeros((rows, nb, 4), dtype=np.uint64)
    ctr[..., 0] = np.arange(nb, dtype=np.uint64)[None, :]
    ctr[..., 1] = np.arange(row0, row0 + rows, dtype=np.uint64)[:, None]
    ctr[..., 2] = np.uint64(site)
    ctr[..., 3] = np.uint64(STREAM_DROPOUT)
    words = philox.philox4x32_10(ctr, philox._key(seed))                   # [rows, nb, 4]
    out = np.empty((rows, nb, 4, 2), dtype=np.uint16)
    out[..., 0] = words & np.uint32(0xFFFF)
    out[..., 1] = words >> np.uint32(16)
    return out.reshape(rows, 8 * nb)[:, :n]


def dropout_factors(seed, site, rows, n, p, row0=0):
    """What dropout multiplies element (r, c) by (0 for a dropped one): float64 [rows, n]."""
    q = int(np.floor(65536.0 * float(np.float32(p)) + 0.5))
    if q == 0:
        return np.ones((rows, n))
    kept = dropout_bits(seed, site, rows, n, row0) >= q
    return np.where(kept, 65536.0 / (65536 - q) if q < 65536 else 0.0, 0.0)


def dropout(x, seed, site, p, res=None):
    """res + dropout(x); a dropped element counts as 0 whatever it was."""
    x = as_f64(x)
    f = dropout_factors(seed, site, x.size // x.shape[-1], x.shape[-1], p).reshape(x.shape)
    out = np.where(f != 0.0, np.where(f != 0.0, x, 0.0) * f, 0.0)
    return out if res is None else out + as_f64(res)


def norm(s, weight=None, bias=None, eps=1e-5, rms=False):
    """(y, mean, rstd) of the rows of s: mean [B*T] (None for RMS), rstd [B*T]."""
    s = as_f64(s)
    n = s.shape[-1]
    w = np.ones(n) if weight is None else as_f64(weight)
    b = np.zeros(n) if bias is None else as_f64(bias)
    eps = float(np.float32(eps))
    mean = np.zeros(s.shape[:-1]) if rms else s.sum(-1) / n
    d = s - mean[..., None]
    rstd = 1.0 / np.sqrt((d * d).sum(-1) / n + eps)
    y = d * rstd[..., None] * w + b
    return y, None if rms else mean.reshape(-1), rstd.reshape(-1)


def norm_backward(dy, s, weight, mean, rstd, ds=None):
    """(dx, dw, db) with the statistics given (mean None: RMS); dw, db [B, n]: each sample's own."""
    dy, s = as_f64(dy), as_f64(s)
    n = s.shape[-1]
    w = np.ones(n) if weight is None else as_f64(weight)
    r = as_f64(rstd).reshape(s.shape[:-1] + (1,))
    xh = (s if mean is None else s - as_f64(mean).reshape(s.shape[:-1] + (1,))) * r
    g = dy * w
    dx = g - xh * ((g * xh).sum(-1, keepdims=True) / n)
    if mean is not None:
        dx = dx - g.sum(-1, keepdims=True) / n
    dx = dx * r
    if ds is not None:
        dx = dx + as_f64(ds)
    return dx, (dy * xh).sum(1), dy.sum(1)


def norm_vectors(G):
    """Squared norm of every sample's vector: [B]."""
    return (as_f64(G) ** 2).sum(1)


def clip_accumulate_vectors(G, c):
    """sum_i c_i G_i over the samples with c_i != 0: [n]."""
    G, c = as_f64(G), as_f64(c)
    out = np.zeros(G.shape[1])
    for i in range(G.shape[0]):
        if c[i] != 0.0:
            out += c[i] * G[i]
    return out
