"""Performance cases of the block-junction operators: dropout, residual sum and norm, and the
private gradients of the norm's own weight and bias.

Between two linear layers of a decoder block lie a dropout, a residual sum and a norm.  A private
training run needs them forwards and backwards, and the gradient of the norm's weight and bias for
every sample by itself, because that is what is clipped: its squared norms join the linear layers'
estimates, its clipped sum joins the private gradient.  Serving needs the forward pass for single
tokens.  The cases take the widths of the repository's workloads (hidden 2048, MLP 8192, 16 blocks,
33 norms) or generic ones (odd widths and lengths, fp32 rows).

``own`` false computes the operators in elementary torch operations, ``own`` true through the
library.  Dropout's mask is a function of (seed, site, row, column): Philox4x32-10 of the counter
(column div 8, row, site, 4) gives 16 bits for each of 8 columns, and an element is dropped when
its 16 bits lie below floor(65536 p + 1/2).
"""

import math

import numpy as np
import torch

own = False

EPS = 1e-5
SITE = 5


def listed():
    return [
        # A small model's fp32 residual junction, odd in every size: only the call's latency counts.
        dict(name="dropout_odd_f32", op="dropout", B=3, T=61, n=111, pad=0, dtype="f32", res=True, p=0.1),
        # The residual junction of a decoder stack in training: the largest stream.
        dict(name="dropout_stack", op="dropout", B=8, T=4096, n=2048, pad=0, dtype="bf16", res=True, p=0.1),
        # Serving one token: residual sum and RMS norm, one row.
        dict(name="norm_token", op="norm", kind="rms", B=1, T=1, n=2048, pad=0, dtype="bf16", res=True, p=0.0,
             bias=False, stats=False),
        # Serving a batch of 64 sequences, one token each, at the MLP's width.
        dict(name="norm_serving", op="norm", kind="rms", B=64, T=1, n=8192, pad=0, dtype="bf16", res=True, p=0.0,
             bias=False, stats=False),
        # An fp32 layer norm by itself (embedding or final norm), odd length and width.
        dict(name="norm_odd_f32", op="norm", kind="layer", B=4, T=1021, n=1111, pad=0, dtype="f32", res=False, p=0.0,
             bias=True, stats=True),
        # The whole junction of a decoder stack in training: dropout, residual sum, layer norm.
        dict(name="norm_stack", op="norm", kind="layer", B=8, T=4096, n=2048, pad=0, dtype="bf16", res=True, p=0.1,
             bias=True, stats=True),
        # The backward pass of a small fp32 model: launches and latency.
        dict(name="backward_small_f32", op="backward", kind="layer", B=2, T=64, n=64, pad=0, dtype="f32", res=False,
             p=0.0),
        # Short samples of an odd length and width, rows on 2-byte boundaries.
        dict(name="backward_odd", op="backward", kind="layer", B=16, T=333, n=1111, pad=3, dtype="bf16", res=True,
             p=0.1),
        # The junction of a decoder stack backwards: dx, the dropped branch's gradient, weight and bias per sample.
        dict(name="backward_stack", op="backward", kind="layer", B=8, T=4096, n=2048, pad=0, dtype="bf16", res=True,
             p=0.1),
        # One sample of long context through an RMS norm: the weight's gradient sums 32768 tokens.
        dict(name="backward_long", op="backward", kind="rms", B=1, T=32768, n=2048, pad=0, dtype="bf16", res=True,
             p=0.0),
        # The private side of a step: squared norms and clipped sums of all 33 RMS norms' weight gradients.
        dict(name="private_step", op="private", B=8, n=33 * 2048, pad=0),
        # The same for layer norms with biases and a large batch of short samples.
        dict(name="private_batch", op="private", B=256, n=33 * 4096, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above: widths, lengths, batches, types, row strides, dropout rates."""
    op = rng.choice(["dropout", "dropout", "norm", "norm", "norm", "backward", "backward", "backward", "private"])
    if op == "private":
        while True:
            B, n = _log_int(rng, 1, 256), _log_int(rng, 256, 33 * 4096)
            if B * n >= 2048:
                return dict(op=op, B=B, n=n, pad=rng.choice([0, 0, 1, 4]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    most = (64 if dtype == "bf16" else 32) << 20
    serving = op == "norm" and rng.random() < 0.4
    while True:
        n = _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            n = n // 64 * 64
        B = _log_int(rng, 1, 64)
        T = 1 if serving else _log_int(rng, 16, 32768)
        if B * T * n <= most:
            break
    case = dict(op=op, B=B, T=T, n=n, pad=rng.choice([0, 0, 0, 3, 8]), dtype=dtype, res=rng.random() < 0.7,
                p=0.0 if serving else rng.choice([0.05, 0.1, 0.1, 0.25, 0.5]))
    if op != "dropout":
        case["kind"] = rng.choice(["layer", "rms"])
        if rng.random() < 0.4:
            case["p"] = 0.0
    if op == "norm":
        case.update(bias=rng.random() < 0.5, stats=not serving)
    return case


# ---- inputs -------------------------------------------------------------------------------------

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1_000_003 + int(stream))


def _rows(case, seed, stream, scale=1.0, offset=None):
    """Token rows [B, T, n] of N(0, scale^2) (scale a number or per sample), rows ``pad`` elements apart."""
    B, T, n = case["B"], case["T"], case["n"]
    x = torch.randn(B, T, n + case["pad"], generator=_gen(seed, stream), device="cuda", dtype=_DTYPES[case["dtype"]])
    x.mul_(scale)
    x = x[:, :, :n]
    if offset is not None:
        x.add_(offset)
    return x


def _lengths(case, seed):
    """True for a sample's real tokens: the last quarter of a batch's lengths is padding in places."""
    B, T = case["B"], case["T"]
    frac = 0.75 + 0.25 * torch.rand(B, 1, generator=_gen(seed, 1), device="cuda")
    return torch.arange(T, device="cuda").view(1, T) < (frac * T).ceil()


def prepare(case, seed):
    B, n = case["B"], case["n"]
    if case["op"] == "private":
        # gradients of lognormal scale over the samples, and clip factors of which a few are 0 (dropped) or 1
        g = torch.randn(B, n + case["pad"], generator=_gen(seed, 2), device="cuda")
        g.mul_(0.01 * torch.exp(torch.randn(B, 1, generator=_gen(seed, 3), device="cuda")))
        c = (1.5 * torch.rand(B, generator=_gen(seed, 4), device="cuda") - 0.1).clamp_(0.0, 1.0)
        return dict(case, G=g[:, :n], c=c)
    dt = _DTYPES[case["dtype"]]
    state = dict(case, seed=(int(seed) * 0x9E3779B97F4A7C15 + 11) % 2 ** 64)
    # a residual stream has features with offsets of their own; a branch's output is smaller than it
    offset = 0.5 * torch.randn(n, generator=_gen(seed, 5), device="cuda").to(dt)
    if case["op"] == "backward":
        s = _rows(case, seed, 6, 1.5, offset)
        real = _lengths(case, seed).view(B, -1, 1)
        scale = 0.01 * torch.exp(torch.randn(B, 1, 1, generator=_gen(seed, 7), device="cuda")).to(dt)
        state.update(s=s, dy=_rows(case, seed, 8, scale).mul_(real.to(dt)),
                     ds=_rows(case, seed, 9, scale).mul_(real.to(dt)) if case["res"] else None)
        sf = s.float()
        mu = sf.mean(-1, keepdim=True) if case["kind"] == "layer" else torch.zeros_like(sf[:, :, :1])
        rstd = ((sf - mu).square().mean(-1, keepdim=True) + EPS).rsqrt()
        state.update(mean=mu.view(-1) if case["kind"] == "layer" else None, rstd=rstd.view(-1))
    else:
        state.update(x=_rows(case, seed, 6, 0.5), res=_rows(case, seed, 8, 1.5, offset) if case["res"] else None)
    if case["op"] != "dropout":
        state["w"] = (1.0 + 0.1 * torch.randn(n, generator=_gen(seed, 10), device="cuda")).to(dt)
        state["b"] = 0.1 * torch.randn(n, generator=_gen(seed, 11), device="cuda").to(dt) if case.get("bias") else None
    return state


# ---- the library ----------------------------------------------------------------------------------

def _run_own(state):
    from paper_2605_24879_amd import dprc as D
    op = state["op"]
    if op == "private":
        return dict(n2=D.dprc_norm_vectors(state["G"]), grad=D.dprc_clip_accumulate_vectors(state["G"], state["c"]))
    if op == "dropout":
        return dict(out=D.dprc_dropout(state["x"], state["p"], state["seed"], SITE, res=state["res"]))
    kind = {"layer": D.LAYERNORM, "rms": D.RMSNORM}[state["kind"]]
    if op == "norm":
        y, s, mean, rstd = D.dprc_layernorm(state["x"], state["w"], state["b"], eps=EPS, kind=kind, res=state["res"],
                                            p=state["p"], seed=state["seed"], site_id=SITE, stats=state["stats"])
        return _norm_outputs(state, y, s, mean, rstd)
    dx, dh, dw, db = D.dprc_layernorm_backward(state["dy"], state["s"], state["w"], state["mean"], state["rstd"],
                                               kind=kind, ds=state["ds"], p=state["p"], seed=state["seed"],
                                               site_id=SITE, bias_grad=state["kind"] == "layer")
    return _backward_outputs(state, dx, dh, dw, db)


def _norm_outputs(state, y, s, mean, rstd):
    out = dict(y=y)
    if state["res"] is not None or state["p"] > 0.0:
        out["s"] = s                                   # otherwise the input itself
    if state["stats"]:
        out["rstd"] = rstd
        if state["kind"] == "layer":
            out["mean"] = mean
    return out


def _backward_outputs(state, dx, dh, dw, db):
    out = dict(dx=dx, dw=dw)
    if state["p"] > 0.0:
        out["dh"] = dh
    if state["kind"] == "layer":
        out["db"] = db
    return out


# ---- the plain form -------------------------------------------------------------------------------

_LOW = 0xFFFFFFFF


def _plain_mask(rows, n, p, seed, device):
    """(kept [rows, n], factor): the Philox rounds on 64-bit integers, all blocks at once."""
    thr = math.floor(65536.0 * p + 0.5)
    nb = (n + 7) // 8
    c0 = torch.arange(nb, device=device).view(1, nb).expand(rows, nb)
    c1 = torch.arange(rows, device=device).view(rows, 1).expand(rows, nb)
    c2 = torch.full((1, 1), SITE, device=device, dtype=torch.int64).expand(rows, nb)
    c3 = torch.full((1, 1), 4, device=device, dtype=torch.int64).expand(rows, nb)
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=-1)
    kept = halves.view(rows, nb * 8)[:, :n] >= thr
    return kept, 65536.0 / (65536 - thr) if thr < 65536 else 0.0


def _plain_drop(x, state):
    if state["p"] == 0.0:
        return x
    B, T, n = x.shape
    kept, factor = _plain_mask(B * T, n, state["p"], state["seed"], x.device)
    return torch.where(kept.view(B, T, n), x * factor, torch.zeros((), device=x.device))


def _run_plain(state):
    op = state["op"]
    if op == "private":
        G, c = state["G"], state["c"]
        return dict(n2=(G * G).sum(1), grad=(G * c.view(-1, 1)).sum(0))
    dt = _DTYPES[state["dtype"]]
    if op == "dropout":
        out = _plain_drop(state["x"].float(), state)
        return dict(out=(out if state["res"] is None else out + state["res"].float()).to(dt))
    layer = state["kind"] == "layer"
    if op == "norm":
        s = _plain_drop(state["x"].float(), state)
        if state["res"] is not None:
            s = s + state["res"].float()
        mean = s.mean(-1, keepdim=True) if layer else 0.0
        rstd = 1.0 / torch.sqrt(((s - mean) ** 2).mean(-1, keepdim=True) + EPS)
        y = (s - mean) * rstd * state["w"].float()
        if state["b"] is not None:
            y = y + state["b"].float()
        return _norm_outputs(state, y.to(dt), s.to(dt), mean.view(-1) if layer else None, rstd.view(-1))
    dy, s = state["dy"].float(), state["s"].float()
    B, T, n = s.shape
    rstd = state["rstd"].view(B, T, 1)
    xh = (s - state["mean"].view(B, T, 1)) * rstd if layer else s * rstd
    g = dy * state["w"].float()
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    if layer:
        dx = dx - g.mean(-1, keepdim=True)
    dx = dx * rstd
    if state["ds"] is not None:
        dx = dx + state["ds"].float()
    dh = _plain_drop(dx, state).to(dt) if state["p"] > 0.0 else None
    return _backward_outputs(state, dx.to(dt), dh, (dy * xh).sum(1), dy.sum(1) if layer else None)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    B, n = case["B"], case["n"]
    if case["op"] == "private":
        return {"bytes": 4 * (2 * B * n + n + 2 * B), "flops": 4 * B * n}
    e = 2 if case["dtype"] == "bf16" else 4
    rows = B * case["T"]
    drop = case["p"] > 0.0
    if case["op"] == "dropout":
        tensors, flops, extra = 2 + case["res"], 2, 0
    elif case["op"] == "norm":
        layer = case["kind"] == "layer"
        tensors = 2 + case["res"] + (case["res"] or drop)
        flops = 8
        extra = n * e * (1 + case["bias"]) + (4 * rows * (1 + layer) if case["stats"] else 0)
    else:
        layer = case["kind"] == "layer"
        tensors, flops = 3 + case["res"] + drop, 14
        extra = n * e + 4 * rows * (1 + layer) + 4 * B * n * (1 + layer)
    return {"bytes": tensors * rows * n * e + extra, "flops": flops * rows * n}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _exact_factors(rows, n, p, seed):
    """What dropout multiplies each element by, from numpy's unsigned 64-bit products, row blocks at a time."""
    below = int(p * 65536 + 0.5)
    if below == 0:
        return None
    out = np.empty((rows, n), dtype=np.float32)
    cols = np.arange(-(-n // 8), dtype=np.uint64)[None, :]
    mask, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    step = max(1, (1 << 20) // cols.size)
    for r0 in range(0, rows, step):
        r = np.arange(r0, min(rows, r0 + step), dtype=np.uint64)[:, None]
        shape = (r.size, cols.size)
        ctr = [np.broadcast_to(v, shape).astype(np.uint64) for v in (cols, r, np.uint64(SITE), np.uint64(4))]
        for i in range(10):
            key = [np.uint64((seed + i * 0x9E3779B9) % 2 ** 32), np.uint64(((seed >> 32) + i * 0xBB67AE85) % 2 ** 32)]
            even, odd = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
            ctr = [(odd >> half) ^ ctr[1] ^ key[0], odd & mask, (even >> half) ^ ctr[3] ^ key[1], even & mask]
        bits = np.stack(ctr, axis=-1).astype("<u4").view("<u2").reshape(r.size, -1)[:, :n]
        out[r0:r0 + r.size] = bits >= below
    return torch.from_numpy(out).cuda().double() * (65536.0 / (65536 - below))


def exact(case, seed):
    st = prepare(case, seed)
    f64 = lambda t: None if t is None else t.double()
    if case["op"] == "private":
        G, c = f64(st["G"]), f64(st["c"])
        return dict(n2=torch.linalg.vector_norm(G, dim=1).square(), grad=torch.mv(G.t().contiguous(), c))
    B, T, n = case["B"], case["T"], case["n"]
    factors = _exact_factors(B * T, n, case["p"], st["seed"])
    apply = lambda t: t if factors is None else t * factors.view(B, T, n)
    if case["op"] == "dropout":
        out = apply(f64(st["x"]))
        return dict(out=out if st["res"] is None else out.add_(f64(st["res"])))
    w = f64(st["w"])
    if case["op"] == "norm":
        s = apply(f64(st["x"]))
        if st["res"] is not None:
            s = s + f64(st["res"])
        if case["kind"] == "layer":
            var, mean = torch.var_mean(s, dim=2, correction=0, keepdim=True)
            centred = s - mean
        else:
            mean, centred, var = None, s, (s * s).sum(2, keepdim=True) / n
        rstd = (var + EPS).pow(-0.5)
        y = centred.mul(rstd).mul_(w)
        if st["b"] is not None:
            y += f64(st["b"])
        return _norm_outputs(st, y, s, None if mean is None else mean.flatten(), rstd.flatten())
    # the row's gradient through the Jacobian of the normalised value: with z = w dy,
    # ds += rstd (z - <z, 1> 1 / n - <z, xh> xh / n)
    r = f64(st["rstd"]).view(B, T, 1)
    xh = f64(st["s"])
    if case["kind"] == "layer":
        xh = xh - f64(st["mean"]).view(B, T, 1)
    xh = xh * r
    dy = f64(st["dy"])
    z = dy * w
    dx = z - xh * ((z * xh).sum(2, keepdim=True) / n)
    if case["kind"] == "layer":
        dx -= z.sum(2, keepdim=True) / n
    dx *= r
    if st["ds"] is not None:
        dx += f64(st["ds"])
    dh = apply(dx) if case["p"] > 0.0 else None
    dw = torch.stack([(dy[i] * xh[i]).sum(0) for i in range(B)])
    return _backward_outputs(st, dx, dh, dw, dy.sum(1) if case["kind"] == "layer" else None)
