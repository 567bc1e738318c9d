"""Performance cases of what a private training step leaves between its linear layers and its loss: the
output head's cross entropy with its gradient, rotary positions, and the clipping of a gradient by its
global norm.

The head computes the logits of N = B T tokens over a vocabulary of V in pieces and keeps none of them:
``loss`` gives every token's loss and log-sum-exp, ``backward`` the gradients of the hidden states and of
the weight.  Tokens with a negative target have no loss.  ``rotary`` turns pairs of every head's features
by their position times a frequency, forwards or (as a gradient's) backwards, for q and k in one call.
``clip`` scales a list of gradients by min(1, max_norm / their joint norm).

The cases take the sizes of the repository's workloads (hidden 2048, MLP 8192, 32 query and 8 key/value
heads of width 64, vocabulary 128256, a vocabulary of 50257) or generic ones (odd widths and lengths,
fp32).  ``own`` false computes the operators in elementary torch operations, ``own`` true through the
library.
"""

import math

import torch

own = False

DECODER = [(2048, 2048), (2048, 512), (2048, 512), (2048, 2048), (2048, 8192), (2048, 8192), (8192, 2048)]


def listed():
    return [
        # The loss of a small fp32 model, odd in every size: launches and latency.
        dict(name="loss_small_f32", op="loss", B=2, T=61, d=200, V=1111, pad=0, dtype="f32", ignored=True),
        # Scoring one token each of 64 sequences: the weight is read once and bounds the call.
        dict(name="loss_serving", op="loss", B=64, T=1, d=2048, V=128256, pad=0, dtype="bf16", ignored=False),
        # The loss of a training batch over the whole vocabulary of the Llama-shaped stack.
        dict(name="loss_stack", op="loss", B=2, T=4096, d=2048, V=128256, pad=0, dtype="bf16", ignored=True),
        # The gradient of a small fp32 model's head, odd sizes: launches and latency.
        dict(name="backward_small_f32", op="backward", B=3, T=50, d=136, V=1009, pad=0, dtype="f32", ignored=True),
        # An odd vocabulary at an odd length, hidden rows with a stride of their own.
        dict(name="backward_odd", op="backward", B=4, T=1021, d=1024, V=50257, pad=3, dtype="bf16", ignored=True),
        # The gradient of the stack's head over a training batch: the largest work of all.
        dict(name="backward_stack", op="backward", B=2, T=4096, d=2048, V=128256, pad=0, dtype="bf16", ignored=True),
        # Serving: one new token of each of 64 sequences, far positions of their own, q and k.
        dict(name="rotary_serving", op="rotary", B=64, T=1, heads=32, kv_heads=8, D=64, r=32, interleaved=False,
             inverse=False, far=True, fused=True, heads_first=False, dtype="bf16", out="bf16", scale=1.0),
        # Pairs side by side over part of an odd head, fp32, backwards, scaled for long contexts.
        dict(name="rotary_part_f32", op="rotary", B=3, T=1021, heads=12, kv_heads=4, D=80, r=20, interleaved=True,
             inverse=True, far=True, fused=False, heads_first=False, dtype="f32", out="f32", scale=1.2),
        # A training batch of the stack: q and k out of one fused buffer, into the order attention reads.
        dict(name="rotary_stack", op="rotary", B=8, T=4096, heads=32, kv_heads=8, D=64, r=32, interleaved=False,
             inverse=False, far=False, fused=True, heads_first=True, dtype="bf16", out="bf16", scale=1.0),
        # The gradients of a small fp32 model, most of them vectors of odd lengths: launches and latency.
        dict(name="clip_small", op="clip", shapes="111x64,64,64x111,111,37,1009x64", dtype="f32", active=True),
        # bf16 gradients of two decoder layers of an odd width.
        dict(name="clip_odd_bf16", op="clip", shapes=",".join(["1111x1111"] * 8 + ["1111x4001"] * 6 + ["1111"] * 4),
             dtype="bf16", active=True),
        # The fp32 gradients of four decoder layers and their norms.
        dict(name="clip_stack", op="clip", shapes=",".join(["%dx%d" % s for s in DECODER] * 4 + ["2048"] * 9),
             dtype="f32", active=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above: tokens, widths, vocabularies, types, layouts, lists of tensors."""
    op = rng.choice(["loss", "loss", "backward", "backward", "rotary", "rotary", "rotary", "clip", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("loss", "backward"):
        serving = op == "loss" and rng.random() < 0.4
        most = 8192 * 2048 * 128256 // (1 if dtype == "bf16" else 16)
        while True:
            d, V = _log_int(rng, 64, 4096), _log_int(rng, 256, 131072)
            if rng.random() < 0.5:
                d, V = d // 64 * 64, V // 64 * 64
            B = _log_int(rng, 1, 128 if serving else 16)
            T = 1 if serving else _log_int(rng, 16, 8192)
            if B * T * d * V <= most and B * T <= 16384:
                break
        return dict(op=op, B=B, T=T, d=d, V=V, pad=rng.choice([0, 0, 3, 8]), dtype=dtype, ignored=not serving)
    if op == "rotary":
        while True:
            D = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
            r = rng.choice([D // 2, D // 2, D // 4, D // 8 + 1])
            kv = _log_int(rng, 1, 16)
            heads = kv * rng.choice([1, 2, 4, 8])
            B = _log_int(rng, 1, 64)
            T = 1 if rng.random() < 0.3 else _log_int(rng, 16, 32768)
            if B * T * (heads + kv) * D <= 8 * 4096 * 40 * 64:
                break
        return dict(op=op, B=B, T=T, heads=heads, kv_heads=kv, D=D, r=r, interleaved=rng.random() < 0.4,
                    inverse=rng.random() < 0.4, far=rng.random() < 0.5, fused=rng.random() < 0.5,
                    heads_first=rng.random() < 0.4, dtype=dtype, out=dtype if rng.random() < 0.6 else
                    rng.choice(["bf16", "f32"]), scale=rng.choice([1.0, 1.0, 1.2]))
    while True:
        shapes = []
        for _ in range(_log_int(rng, 1, 60)):
            if rng.random() < 0.4:
                shapes.append((_log_int(rng, 1, 8192),))
            else:
                shapes.append((_log_int(rng, 16, 8192), _log_int(rng, 16, 8192)))
        total = sum(math.prod(s) for s in shapes)
        if 1024 <= total <= 240_000_000:
            break
    return dict(op=op, shapes=",".join("x".join(map(str, s)) for s in shapes), dtype=dtype, active=rng.random() < 0.7)


# ---- inputs -------------------------------------------------------------------------------------

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1_000_003 + int(stream))


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")]


def _prepare_head(case, seed):
    B, T, d, V, dt = case["B"], case["T"], case["d"], case["V"], _DTYPES[case["dtype"]]
    W = (torch.randn(V, d, generator=_gen(seed, 1), device="cuda") * (0.9 / math.sqrt(d))).to(dt)
    target = torch.randint(0, V, (B, T), generator=_gen(seed, 2), device="cuda")
    # hidden states lean towards their target's row by as much as a trained model's do: its probability
    # lies anywhere from 1 / V to about a half
    lean = torch.rand(B, T, 1, generator=_gen(seed, 3), device="cuda") * (math.log(V) / 0.81)
    h = torch.randn(B, T, d + case["pad"], generator=_gen(seed, 4), device="cuda")
    h[:, :, :d] += lean * W[target].float()
    h = h.to(dt)[:, :, :d]
    if case["ignored"]:                                # padding at the end of the samples has no target
        frac = 0.75 + 0.25 * torch.rand(B, 1, generator=_gen(seed, 5), device="cuda")
        target = torch.where(torch.arange(T, device="cuda").view(1, T) < (frac * T).ceil(), target, -100)
    state = dict(case, h=h, W=W, target=target)
    if case["op"] == "backward":
        rows = h.reshape(B * T, d)
        lse = torch.cat([torch.logsumexp(x.float() @ W.float().t(), dim=1) for x in rows.split(1024)])
        # the gradient of the samples' mean losses, weighted as a step weights its samples
        weight = torch.exp(torch.randn(B, 1, generator=_gen(seed, 6), device="cuda"))
        state.update(lse=lse.view(B, T), g=(weight / T).expand(B, T).contiguous())
    return state


def _prepare_rotary(case, seed):
    B, T, H, K, D, dt = (case[k] for k in ("B", "T", "heads", "kv_heads", "D", "dtype"))
    dt = _DTYPES[dt]
    if case["fused"]:                                  # q, k and v of one product, heads side by side
        rows = torch.randn(B, T, H + 2 * K, D, generator=_gen(seed, 1), device="cuda").to(dt)
        q, k = rows[:, :, :H], rows[:, :, H:H + K]
    else:
        q = torch.randn(B, T, H, D, generator=_gen(seed, 1), device="cuda").to(dt)
        k = torch.randn(B, T, K, D, generator=_gen(seed, 2), device="cuda").to(dt)
    r = case["r"]
    j = torch.arange(r, device="cuda", dtype=torch.float64)
    freqs = torch.pow(torch.tensor(500000.0, device="cuda", dtype=torch.float64), -j / r)
    if case["scale"] != 1.0:
        # scaled for long contexts: slow pairs turn by an eighth, with a ramp from the fast ones
        freqs = freqs * (1.0 - 0.875 * ((j / r - 0.3) / 0.4).clamp(0.0, 1.0))
    pos = None
    if case["far"]:
        start = torch.randint(0, 1_000_000, (B, 1), generator=_gen(seed, 3), device="cuda")
        pos = start + torch.arange(T, device="cuda").view(1, T)
    return dict(case, q=q, k=k, freqs=freqs, pos=pos)


def _prepare_clip(case, seed):
    dt = _DTYPES[case["dtype"]]
    shapes = _shapes(case)
    grads = []
    for i, s in enumerate(shapes):                     # layers' gradients differ in scale
        g = torch.randn(s, generator=_gen(seed, 10 + i), device="cuda", dtype=dt)
        grads.append(g.mul_(10.0 ** (-3 + 2 * math.sin(i + seed % 7))))
    total = math.sqrt(sum(math.prod(s) * 10.0 ** (-6 + 4 * math.sin(i + seed % 7)) for i, s in enumerate(shapes)))
    return dict(case, grads=grads, outs=[torch.empty_like(g) for g in grads],
                max_norm=total * (0.3 if case["active"] else 2.0))


def prepare(case, seed):
    if case["op"] in ("loss", "backward"):
        return _prepare_head(case, seed)
    return (_prepare_rotary if case["op"] == "rotary" else _prepare_clip)(case, seed)


# ---- the library ----------------------------------------------------------------------------------

def _run_own(state):
    from paper_2605_24879_amd import dprc as D
    op = state["op"]
    if op == "loss":
        loss, lse = D.dprc_head_loss(state["h"], state["W"], state["target"])
        return dict(loss=loss, lse=lse)
    if op == "backward":
        dh, dW = D.dprc_head_backward(state["h"], state["W"], state["target"], state["lse"], state["g"])
        return dict(dh=dh, dW=dW)
    if op == "rotary":
        q, k = D.dprc_rotary([state["q"], state["k"]], state["freqs"], pos=state["pos"], scale=state["scale"],
                             interleaved=state["interleaved"], inverse=state["inverse"],
                             heads_first=state["heads_first"], out_dtype=_DTYPES[state["out"]])
        return dict(q=q, k=k)
    outs, norm = D.dprc_grad_clip(state["grads"], state["max_norm"], outs=state["outs"])
    return dict(outs=outs, norm=norm)


# ---- the plain form -------------------------------------------------------------------------------

def _plain_head(state):
    B, T, d = state["h"].shape
    h, W = state["h"].float().reshape(B * T, d), state["W"].float()
    target = state["target"].reshape(-1)
    kept, at = target >= 0, target.clamp(min=0).view(-1, 1)
    logits = h @ W.t()
    if state["op"] == "loss":
        top = logits.max(dim=1, keepdim=True).values
        lse = top + torch.log(torch.exp(logits - top).sum(dim=1, keepdim=True))
        loss = torch.where(kept, (lse - logits.gather(1, at)).view(-1), torch.zeros((), device=h.device))
        return dict(loss=loss.view(B, T), lse=lse.view(B, T))
    lse, g = state["lse"].reshape(-1, 1), torch.where(kept, state["g"].reshape(-1), torch.zeros((), device=h.device))
    E = torch.exp(logits.sub_(lse))
    E.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    E.mul_(g.view(-1, 1))
    dt = _DTYPES[state["dtype"]]
    return dict(dh=(E @ W).to(dt).view(B, T, d), dW=(E.t() @ h).to(dt))


def _plain_rotary(x, state, cos, sin):
    D, r = state["D"], state["r"]
    x = x.float()
    if state["interleaved"]:
        a, b = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
    else:
        a, b = x[..., :r], x[..., r:2 * r]
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], dim=-1).flatten(-2) if state["interleaved"] else torch.cat([c, d], dim=-1)
    out = torch.cat([turned, x[..., 2 * r:]], dim=-1) if 2 * r < D else turned
    out = out.to(_DTYPES[state["out"]])
    return out.transpose(1, 2).contiguous().transpose(1, 2) if state["heads_first"] else out


def _run_plain(state):
    op = state["op"]
    if op in ("loss", "backward"):
        return _plain_head(state)
    if op == "rotary":
        B, T = state["B"], state["T"]
        pos = state["pos"] if state["pos"] is not None else torch.arange(T, device="cuda").view(1, T).expand(B, T)
        angle = pos.double().view(B, T, 1, 1) * state["freqs"]
        cos, sin = (state["scale"] * torch.cos(angle)).float(), (state["scale"] * torch.sin(angle)).float()
        if state["inverse"]:
            sin = -sin
        return dict(q=_plain_rotary(state["q"], state, cos, sin), k=_plain_rotary(state["k"], state, cos, sin))
    squares = [g.float().square().sum(dtype=torch.float64) for g in state["grads"]]
    norm = torch.stack(squares).sum().sqrt()
    c = (state["max_norm"] / norm).clamp(max=1.0).float()
    outs = [torch.mul(g.float(), c).to(g.dtype) for g in state["grads"]]
    return dict(outs=outs, norm=norm.float().view(1))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    if case["op"] == "clip":
        n, e = sum(math.prod(s) for s in _shapes(case)), 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * e + 4, "flops": 3 * n}
    if case["op"] == "rotary":
        rows = case["B"] * case["T"]
        n = rows * (case["heads"] + case["kv_heads"])
        e = sum(2 if case[k] == "bf16" else 4 for k in ("dtype", "out"))
        return {"bytes": n * case["D"] * e + 8 * case["r"] + (8 * rows if case["far"] else 0),
                "flops": 6 * n * case["r"]}
    N, d, V, e = case["B"] * case["T"], case["d"], case["V"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "loss":
        return {"bytes": (N + V) * d * e + 16 * N, "flops": 2 * N * d * V}
    return {"bytes": 2 * (N + V) * d * e + 16 * N, "flops": 6 * N * d * V}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _exact_head(case, st):
    """Token blocks at a time, every vector of logits whole, in float64."""
    B, T, d = case["B"], case["T"], case["d"]
    W = st["W"].double()
    rows, target = st["h"].double().reshape(B * T, d), st["target"].reshape(-1)
    Wt = W.t().contiguous()
    if case["op"] == "loss":
        loss, lse = [], []
        for x, y in zip(rows.split(2048), target.split(2048)):
            l = torch.mm(x, Wt)
            z = torch.logsumexp(l, dim=1)
            lse.append(z)
            picked = l[torch.arange(len(y), device=l.device), y.clamp(min=0)]
            loss.append(torch.where(y < 0, torch.zeros_like(z), z - picked))
        return dict(loss=torch.cat(loss).view(B, T), lse=torch.cat(lse).view(B, T))
    lse, g = st["lse"].double().reshape(-1), st["g"].double().reshape(-1)
    dh, dW = [], torch.zeros_like(W)
    for x, y, z, w in zip(rows.split(2048), target.split(2048), lse.split(2048), g.split(2048)):
        p = torch.mm(x, Wt).sub_(z[:, None]).exp_()
        real = torch.nonzero(y >= 0).view(-1)
        p[real, y[real]] -= 1.0
        p *= torch.where(y < 0, torch.zeros_like(w), w)[:, None]
        dh.append(torch.mm(p, W))
        dW += torch.mm(p.t().contiguous(), x)
    return dict(dh=torch.cat(dh).view(B, T, d), dW=dW)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("loss", "backward"):
        return _exact_head(case, st)
    if case["op"] == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in st["grads"]]))
        c = min(1.0, st["max_norm"] / norm.item())
        return dict(outs=[g.double() * c for g in st["grads"]], norm=norm.view(1))
    B, T, D, r = case["B"], case["T"], case["D"], case["r"]
    pos = st["pos"] if st["pos"] is not None else torch.arange(T, device="cuda").expand(B, T)
    # as products of complex numbers of modulus `scale`
    angle = pos.double()[:, :, None, None] * st["freqs"][None, None, None, :]
    turn = torch.polar(torch.full_like(angle, case["scale"]), -angle if case["inverse"] else angle)
    out = {}
    for name in ("q", "k"):
        y = st[name].double().contiguous()
        first = slice(0, 2 * r, 2) if case["interleaved"] else slice(0, r)
        second = slice(1, 2 * r, 2) if case["interleaved"] else slice(r, 2 * r)
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out
