"""Host logic of the head module, rotary positions and the joint clipping in the private training step (no GPU): the
library's calls are played by the oracle on host tensors, so the step's own bookkeeping is what is tested.

The estimates of the layers and the head are their exact squared norms here.
"""

import math

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import head as O
from oracle import junction as J
from paper_2605_24879_amd import dprc, dpsgd, head, rotary
from workloads import llama

SIZES = dict(layers=2, hidden=16, mlp=24, heads=4, kv_heads=2, vocab=19)
f32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float()
f64 = est.as_f64
calls = []


def E_of(h, W, target, lse, g):
    return O.errors(f64(h), f64(W), target.numpy(), f64(lse), f64(g))


def head_loss(h, W, target):
    return tuple(f32(x) for x in O.loss(f64(h), f64(W), target.numpy()))


def head_backward(h, W, target, lse, g, hidden_grad=True, weight_grad=True, k=0, seed=0, layer_id=0, side=0, probe=0):
    calls.append((seed, layer_id, k, hidden_grad))
    E = E_of(h, W, target, lse, g)
    dh = f32(E @ f64(W)) if hidden_grad else None
    dW = f32(np.einsum("btv,btd->vd", E, f64(h))) if weight_grad else None
    return (dh, dW) if k == 0 else (dh, dW, f32([((f64(h)[i].T @ E[i]) ** 2).sum() for i in range(len(E))]))


def head_clip_accumulate(h, W, target, lse, g, c):
    return f32(est.clip_accumulate(f64(h), E_of(h, W, target, lse, g), f64(c)))


def grad_clip(tensors, max_norm, outs=None):
    ys, norm = O.clip([f64(t) for t in tensors], max_norm)
    for t, y in zip(tensors, ys):
        t.copy_(f32(y))
    return tensors, f32([norm])


def rotate(xs, freqs, pos=None, start=0, scale=1.0, interleaved=False, inverse=False, heads_first=False, out_dtype=None):
    out = []
    for x in xs:
        B, T = x.shape[:2]
        p = pos.numpy() if pos is not None else np.broadcast_to(start + np.arange(T), (B, T))
        out.append(torch.from_numpy(O.rotary(f64(x), freqs.numpy(), p, scale, interleaved, inverse)).to(out_dtype or x.dtype))
    return out


def sample_norms(pairs):
    return sum(np.array([((f64(A[i]).T @ f64(E[i])) ** 2).sum() for i in range(len(A))]) for (A, E, _) in pairs)


def norm_hutch_clip(pairs, k, seed, C, side=0, probe=0, n2=None, accumulate=False):
    n2 = f32(sample_norms(pairs) + (f64(n2) if accumulate else 0.0))
    return n2, f32(est.clip_scale(f64(n2), C))


def adamw(theta, m, v, G, sigma, C, seed, tensor_id, inv_batch, lr, beta1, beta2, eps, weight_decay, step, w=None):
    calls.append(("adamw", tensor_id, sigma))
    g = f32(est.add_noise(f64(G), sigma, C, seed, tensor_id)) * inv_batch
    m.mul_(beta1).add_((1 - beta1) * g)
    v.mul_(beta2).add_((1 - beta2) * g * g)
    theta.mul_(1 - lr * weight_decay).sub_(lr * (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps))
    if w is not None and w.dtype == theta.dtype:
        w.copy_(theta.t())


@pytest.fixture(autouse=True)
def library(monkeypatch):
    calls.clear()
    for name, f in dict(
            head_loss=head_loss, head_backward=head_backward, head_clip_accumulate=head_clip_accumulate, grad_clip=grad_clip,
            rotary=rotate, norm_hutch_clip=norm_hutch_clip, private_adamw=adamw,
            clip_scale=lambda n2, C: f32(est.clip_scale(f64(n2), C)), clip_accumulate_workspace=lambda A, E: 0,
            clip_accumulate_layers=lambda pairs, c: [], norm_vectors=lambda G: f32(J.norm_vectors(G)),
            clip_accumulate=lambda A, E, c, ws=None: torch.einsum("btd,b,btp->dp", A, c, E),
            add_noise=lambda g, sigma, C, seed, tensor_id: g.copy_(f32(est.add_noise(f64(g), sigma, C, seed, tensor_id)))).items():
        monkeypatch.setattr(dprc, "dprc_" + name, f)


def stack(seed=3, **kw):
    return llama.build(seed=seed, device="cpu", dtype=torch.float32, **dict(SIZES, head=True, rotary=True, **kw))


def tokens(B=3, seed=1):
    return llama.tokens(B, 7, SIZES["vocab"], seed=seed, device="cpu")


def loss_of(model, tok):
    return lambda: model(tok[:, :-1], tok[:, 1:]).mean(dim=1)


def driver(model, **kw):
    return dpsgd.DPSGDRC(model.linears(), **dict(dict(C=0.5, sigma=0.0, head=model.head), **kw))


def test_the_model_with_them_is_the_plain_one():
    model, plain = stack(), llama.build(seed=3, device="cpu", dtype=torch.float32, **SIZES)
    assert sorted(model.state_dict()) == sorted(plain.state_dict())
    model.load_state_dict(plain.state_dict())
    tok = tokens()
    a, b = llama.per_sample_loss(plain(tok[:, :-1]), tok[:, 1:]), loss_of(model, tok)()
    assert torch.allclose(a, b, rtol=1e-5)
    with torch.no_grad():
        assert torch.equal(loss_of(model, tok)(), b)
    ga = torch.autograd.grad(a.sum(), list(plain.parameters()))
    gb = torch.autograd.grad(b.sum(), list(model.parameters()))
    for x, y in zip(ga, gb):
        assert torch.allclose(x, y, rtol=1e-3, atol=1e-6)
    assert len(model.linears()) == len(plain.linears()) - 1
    with pytest.raises(ValueError):
        plain(tok[:, :-1], tok[:, 1:])


def test_capture_has_the_heads_part():
    """Squared norms and clipped sums with the head are those of all layers' per-sample gradients."""
    model, tok = stack(), tokens()
    drv = driver(model)
    losses, pairs = drv.capture(loss_of(model, tok))
    assert model.head.sink is None and calls[-1] == (drv.seed, len(drv.linears), drv.k, True)
    n2, c, grads = drv.private_grads(pairs, dpsgd.step_seed(drv.seed, 0))
    assert len(calls) == 1                                  # the estimates of the capture were the step's
    lins = model.linears() + [model.lm_head]
    rows = [torch.autograd.grad(loss_of(model, tok[i:i + 1])()[0], [m.weight for m in lins]) for i in range(3)]
    want = np.array([sum((f64(g) ** 2).sum() for g in r) for r in rows])
    assert np.allclose(n2.numpy(), want, rtol=1e-4)
    for j, g in enumerate(grads):
        ref = sum(ci * r[j].t() for ci, r in zip(c, rows))
        assert torch.allclose(g, ref, rtol=1e-3, atol=1e-5 * ref.abs().max().item())
    # under another key they are formed again; what a capture returned stands on its own
    other = drv.capture(loss_of(model, tokens(2, 5)))[1]
    n3, _ = drv.estimate(pairs, 77)
    assert calls[-1] == (77, len(drv.linears), drv.k, False) and torch.allclose(n3, n2)
    again = drv.estimate(pairs, dpsgd.step_seed(drv.seed, 0))[0]
    assert torch.equal(again, n2)
    for bad in (list(pairs), dpsgd.Pairs(pairs), dpsgd.Pairs(pairs, head=other.head)):
        with pytest.raises(ValueError):
            drv.estimate(bad, 7)
        with pytest.raises(ValueError):
            drv.clipped_sums(bad, c)
    with torch.no_grad():
        model.lm_head.weight.mul_(1.0)                      # the head's gradients are formed from it again
    with pytest.raises(RuntimeError, match="changed"):
        drv.clipped_sums(pairs, c)
    drv.remove_hooks()


def test_the_head_alone_is_trained():
    model, tok = stack(), tokens()
    drv = dpsgd.DPSGDRC([], C=0.5, sigma=0.0, head=model.head)
    n2, c, grads = drv.private_grads(drv.capture(loss_of(model, tok))[1], 0)
    rows = [torch.autograd.grad(loss_of(model, tok[i:i + 1])()[0], model.lm_head.weight)[0] for i in range(3)]
    assert np.allclose(n2.numpy(), [(f64(g) ** 2).sum() for g in rows], rtol=1e-4)
    assert len(grads) == 1 and torch.allclose(grads[0], sum(ci * g.t() for ci, g in zip(c, rows)), rtol=1e-3, atol=1e-6)
    # targets in a buffer that is filled anew before the clipped sums, and a capture that fails half-way
    x, y = model.norm(model.embed(tok[:, :-1])).detach(), tok[:, 1:].contiguous()
    pairs = drv.capture(lambda: model.head(x, y).mean(1))[1]
    want = drv.clipped_sums(pairs, c)[0]
    y.zero_()
    assert torch.equal(drv.clipped_sums(pairs, c)[0], want)

    def fails():
        torch.autograd.grad(model.head(x, y).sum(), model.lm_head.weight, allow_unused=True)
        raise KeyError
    with pytest.raises(KeyError):
        drv.capture(fails)
    assert drv._head is None and model.head.sink is None
    drv.update(drv.clipped_sums(pairs, c), 3, 0)
    with pytest.raises(RuntimeError, match="changed"):
        drv.estimate(pairs, 0)


def test_what_the_step_refuses():
    model, tok = stack(), tokens()
    with pytest.raises(ValueError):
        dpsgd.DPSGDRC(model.linears() + [model.lm_head], C=1.0, sigma=0.0, head=model.head)
    with pytest.raises(ValueError):
        driver(model, estimator="hutchpp")
    for bad in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(ValueError):
            driver(model, max_norm=bad)
    with pytest.raises(ValueError):
        head.Head(torch.nn.Linear(4, 5))
    drv = driver(model)
    twice = lambda: (model(tok[:, :-1], tok[:, 1:]) + model(tok[:, :-1], tok[:, 1:])).mean(1)
    with pytest.raises(RuntimeError, match="twice"):
        drv.capture(twice)
    assert model.head.sink is None
    with pytest.raises(RuntimeError, match="part"):
        drv.capture(lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]))
    flat = lambda: model.head(torch.cat([s for s in model.norm(model.embed(tok[:, :-1]))])[None], tok[:, 1:].reshape(1, -1)).view(3, -1).mean(1)
    alone = dpsgd.DPSGDRC([], C=1.0, sigma=0.0, head=model.head)
    with pytest.raises(RuntimeError, match="batch"):
        alone.capture(flat)
    drv.remove_hooks()


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("max_norm", [None, 0.05, 100.0])
def test_steps(fused, max_norm):
    """The noise of every layer, the norms and the head is its own; the update is that of the clipped noisy mean."""
    model, tok = stack(junctions=False), tokens()
    drv = driver(model, sigma=0.7, fused_adamw=fused, max_norm=max_norm, lr=0.01)
    _, pairs = drv.capture(loss_of(model, tok))
    _, c, clean = drv.private_grads(pairs, dpsgd.step_seed(drv.seed, 0), noise=False)
    nl = len(drv.linears)
    ids = list(range(nl)) + [nl + 1]
    want = [est.add_noise(f64(g), 0.7, 0.5, dpsgd.step_seed(drv.seed, 0), j) / 3 for g, j in zip(clean, ids)]
    if max_norm is not None:
        want, norm = O.clip(want, max_norm)
    before = [m.clone() for m in drv._masters()]
    calls.clear()
    drv.step(loss_of(model, tok))
    if max_norm is not None:
        assert np.allclose(drv.last["norm"].numpy(), norm, rtol=1e-5)
    if fused:
        assert [x[1:] for x in calls if x[0] == "adamw"] == [(j, 0.7 if max_norm is None else 0.0) for j in ids]
    for b, m, g in zip(before, drv._masters(), want):        # AdamW's first step: lr g / (|g| + eps)
        assert np.allclose(f64(b - m), 0.01 * g / (np.abs(g) + 1e-8), rtol=2e-3, atol=1e-6)
    assert torch.equal(model.lm_head.weight, drv.head_master.t()) and drv.steps == 1
    drv.remove_hooks()


def test_frequencies():
    f, scale = rotary.frequencies(64, 500000.0)
    assert scale == 1.0 and torch.equal(f, 500000.0 ** (-2 * torch.arange(32, dtype=torch.float64) / 64))
    assert torch.allclose(rotary.frequencies(64, scaling=dict(kind="linear", factor=4))[0], rotary.frequencies(64)[0] / 4, rtol=1e-15)
    n = rotary.frequencies(64, scaling=dict(kind="ntk", factor=8))[0]
    assert n[0] == 1.0 and math.isclose(n[-1], rotary.frequencies(64)[0][-1] / 8, rel_tol=1e-12)
    w = rotary.frequencies(64, 500000.0, dict(kind="wavelength", factor=32, low=1, high=4, original=8192))[0]
    length = 2 * math.pi / f
    assert torch.equal(w[length < 2048], f[length < 2048]) and torch.allclose(w[length > 8192], f[length > 8192] / 32, rtol=1e-15)
    mid = (length > 2048) & (length < 8192)
    assert mid.any() and (w[mid] < f[mid]).all() and (w[mid] > f[mid] / 32).all()
    r, a = rotary.frequencies(128, 10000.0, dict(kind="ramp", factor=16, original=4096))
    p = rotary.frequencies(128)[0]
    turns = 4096 * p / (2 * math.pi)
    assert torch.allclose(r[turns > 33], p[turns > 33]) and torch.allclose(r[turns < 0.9], p[turns < 0.9] / 16) and math.isclose(a, 0.1 * math.log(16) + 1)
    for bad in (3, 0):
        with pytest.raises(ValueError):
            rotary.frequencies(bad)
    with pytest.raises(ValueError):
        rotary.frequencies(4, scaling=dict(kind="other", factor=2, original=8))
    with pytest.raises(ValueError):
        rotary.Rotary(64, dim=66)


def test_rotary_module():
    rot = rotary.Rotary(8, dim=6, scaling=dict(kind="ramp", factor=4, original=64))
    assert rot.to(torch.bfloat16).freqs.dtype == torch.float64
    q, k = torch.randn(2, 5, 3, 8, dtype=torch.float64, requires_grad=True), torch.randn(2, 5, 1, 8, dtype=torch.float64, requires_grad=True)
    pos = torch.randint(0, 50, (2, 5))
    a, b = rot(q, k, pos=pos)
    assert np.allclose(a.detach().numpy(), O.rotary(q.detach().numpy(), rot.freqs.numpy(), pos.numpy(), rot.scale))
    # the turn is linear in x: its gradient against the sum of products is exact
    ga, gb = torch.randn_like(a), torch.randn_like(b)
    gq, gk = torch.autograd.grad((a * ga).sum() + (b * gb).sum(), [q, k])
    assert torch.allclose((gq * q).sum() + (gk * k).sum(), (a * ga).sum() + (b * gb).sum())
    assert torch.equal(rot(q.detach(), pos=pos), a.detach()) and not rot(q.detach()).requires_grad
    with pytest.raises(ValueError):
        rot(torch.zeros(1, 1, 1, 6))
    first = rotary.Rotary(8)
    with torch.inference_mode():                            # then trained
        first(torch.zeros(1, 1, 1, 8, dtype=torch.float64))
    torch.autograd.grad(first(q).sum(), q)


def test_tables_are_made_where_they_are_read(monkeypatch):
    """The stack's own cosines and sines are for blocks without a rotary module."""
    made, tables, tok = [], llama._rope_tables, tokens()
    monkeypatch.setattr(llama, "_rope_tables", lambda *a: made.append(a) or tables(*a))
    plain = llama.build(seed=3, device="cpu", dtype=torch.float32, **SIZES)
    loss_of(stack(), tok)()
    assert not made
    plain(tok[:, :-1])
    assert len(made) == 1
