"""Host logic of junctions in the private training step (no GPU): the library's calls are played by
the oracle on host tensors, so the step's own bookkeeping is what is tested.

The estimates of the linear layers are their exact squared norms here.
"""

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import junction as J
from paper_2605_24879_amd import dprc, dpsgd, junction
from workloads import llama

SIZES = dict(layers=2, hidden=16, mlp=24, heads=4, kv_heads=2, vocab=19)
f32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float()


def layernorm(x, weight=None, bias=None, eps=1e-5, kind=dprc.LAYERNORM, res=None, p=0.0, seed=0, site_id=0, stats=True):
    s64 = J.dropout(x, seed, site_id, p, res=res)
    y, mean, rstd = J.norm(s64, weight, bias, eps=eps, rms=kind == dprc.RMSNORM)
    s = x if res is None and p == 0.0 else f32(s64)
    return f32(y), s, None if mean is None else f32(mean), f32(rstd)


def layernorm_backward(dy, s, weight, mean, rstd, kind=dprc.LAYERNORM, ds=None, p=0.0, seed=0, site_id=0, weight_grad=True,
                       bias_grad=True, dw=None, db=None):
    assert (mean is None) == (kind == dprc.RMSNORM)
    dx, w, b = J.norm_backward(dy, s, weight, mean, rstd, ds=ds)
    out = []
    for given, want, g in ((dw, weight_grad, w), (db, bias_grad, b)):
        out.append(f32(g) if given is None and want else given)
        if given is not None:
            assert given.shape == g.shape
            given.copy_(f32(g))
    return f32(dx), f32(J.dropout(dx, seed, site_id, p)) if p > 0.0 else None, *out


def norm_vectors(G):
    return f32(J.norm_vectors(G))


def sample_norms(pairs):
    return sum(np.array([((est.as_f64(A[i]).T @ est.as_f64(E[i])) ** 2).sum() for i in range(len(A))]) for (A, E, _) in pairs)


def norm_hutch_clip(pairs, k, seed, C, side=0, probe=0, n2=None, accumulate=False):
    n2 = f32(sample_norms(pairs) + (est.as_f64(n2) if accumulate else 0.0))
    return n2, f32(est.clip_scale(est.as_f64(n2), C))


def add_noise(g, sigma, C, seed, tensor_id):
    return g.copy_(f32(est.add_noise(est.as_f64(g), sigma, C, seed, tensor_id)))


@pytest.fixture(autouse=True)
def library(monkeypatch):
    for name, f in dict(
            layernorm=layernorm, layernorm_backward=layernorm_backward, norm_vectors=norm_vectors, norm_hutch_clip=norm_hutch_clip,
            dropout=lambda x, p, seed, site_id, res=None: f32(J.dropout(x, seed, site_id, p, res=res)),
            clip_accumulate_vectors=lambda G, c: f32(J.clip_accumulate_vectors(G, c)), clip_accumulate_workspace=lambda A, E: 0,
            clip_accumulate=lambda A, E, c, ws=None: torch.einsum("btd,b,btp->dp", A, c, E), add_noise=add_noise).items():
        monkeypatch.setattr(dprc, "dprc_" + name, f)


def stack(**kw):
    return llama.build(seed=3, device="cpu", dtype=torch.float32, **dict(SIZES, junctions=True, **kw))


def loss_of(model, tok):
    return lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:])


def tokens(B=3, seed=1):
    return llama.tokens(B, 7, SIZES["vocab"], seed=seed, device="cpu")


def driver(model, **kw):
    return dpsgd.DPSGDRC(model.linears(), **dict(dict(C=0.5, sigma=0.0, norms=model.norms()), **kw))


def reference(model, tok):
    """Per-sample gradients of the norms' parameters [B, N], each sample alone through torch's autograd."""
    params = [q for m in model.norms() for q in m.parameters_in_order()]
    rows = [torch.cat([g.reshape(-1) for g in torch.autograd.grad(loss_of(model, tok[i:i + 1])()[0], params)]) for i in range(len(tok))]
    return torch.stack(rows)


def test_each_capture_keeps_its_own_norm_gradients():
    # what a capture returns stands on its own: other captures between it and its use change nothing, and it
    # can be used again
    model = stack(norm="layer")
    drv = driver(model)
    toks = tokens(3, 1), tokens(2, 2)
    refs = [reference(model, t) for t in toks]
    alone = [drv.private_grads(drv.capture(loss_of(model, t))[1], 7) for t in toks]
    both = [drv.capture(loss_of(model, t))[1] for t in toks]
    for use in (0, 1, 0):
        n2, c, grads = drv.private_grads(both[use], 7)
        for a, b in zip((n2, c, *grads), (*alone[use][:2], *alone[use][2])):
            assert torch.equal(a, b)
        G = refs[use]
        want = sample_norms(both[use]) + (G.double() ** 2).sum(1).numpy()
        assert np.all(np.abs(n2.numpy() - want) <= 1e-4 * want)
        assert torch.allclose(grads[-1][0], (c[:, None] * G).sum(0), rtol=1e-3, atol=1e-5 * G.abs().max().item())
    # layers without the norms' gradients beside them are refused, not paired with some capture's
    with pytest.raises(ValueError):
        drv.private_grads(list(both[0]), 7)
    with pytest.raises(ValueError):
        drv.estimate(both[0][:3], 7)
    same = drv.private_grads(dpsgd.Pairs(list(both[0]), both[0].vectors), 7)
    assert torch.equal(same[0], alone[0][0])
    drv.remove_hooks()


class Flattened(torch.nn.Module):
    """A junction that is handed all samples' rows as one sample's."""

    def __init__(self, inner):
        super().__init__()
        self.inner = inner

    def forward(self, x, res=None):
        B, T, n = x.shape
        y, s = self.inner(x.reshape(1, B * T, n), None if res is None else res.reshape(1, B * T, n))
        return y.view(B, T, n), s.view(B, T, n)


def test_norms_that_see_another_batch_are_refused():
    # their per-sample gradients would have one row for three samples, and so would n2
    model = stack()
    norms, tok = model.norms(), tokens()
    for b in model.blocks:
        b.norm1, b.norm2 = Flattened(b.norm1), Flattened(b.norm2)
    model.norm = Flattened(model.norm)
    drv = driver(model, norms=norms)
    with pytest.raises(RuntimeError, match="batch"):
        drv.capture(loss_of(model, tok))
    assert all(m.sink is None for m in norms)
    with pytest.raises(RuntimeError, match="batch"):
        drv.step(loss_of(model, tok))
    drv.remove_hooks()
    model = stack()
    drv = driver(model)
    three, two = (drv.capture(loss_of(model, tokens(B)))[1] for B in (3, 2))
    for f in (lambda pairs: drv.estimate(pairs, 7), lambda pairs: drv.clipped_sums(pairs, torch.ones(3))):
        with pytest.raises(ValueError, match="batch"):
            f(dpsgd.Pairs(three, two.vectors))
    drv.remove_hooks()


@pytest.mark.parametrize("norms", [False, True])
def test_noise_goes_by_the_layer(norms):
    # the noise of a layer is keyed by its number, whichever layers a call has and in whatever order: parts of a
    # step must not share their noise
    model = stack()
    drv = driver(model, sigma=0.7, **({} if norms else dict(norms=())))
    _, pairs = drv.capture(loss_of(model, tokens()))
    nl = len(pairs)
    for order in ([4], [2, 0, 7], list(range(nl))[::-1]):
        part = dpsgd.Pairs([pairs[j] for j in order], pairs.vectors)
        _, c, noisy = drv.private_grads(part, 9)
        for g, clean, j in zip(noisy, drv.clipped_sums(part, c), order + [nl] * norms):
            want = est.add_noise(est.as_f64(clean), 0.7, 0.5, 9, j)
            assert np.max(np.abs(est.as_f64(g) - want)) <= 1e-6 * np.max(np.abs(want)), j
        assert len(noisy) == len(order) + norms
    drv.remove_hooks()


def test_shared_norm_parameters_are_refused():
    # each listed parameter has gradients and a master of its own: one that two modules share would be trained
    # on half of its gradient and count wrongly in the norms
    a, b = junction.Junction(8), junction.Junction(8)
    b.weight = a.weight
    held = a.weight.data_ptr()
    for norms in ([a, b], [a, a]):
        with pytest.raises(ValueError):
            dpsgd.DPSGDRC([], C=1.0, sigma=0.0, norms=norms)
    assert a.weight.data_ptr() == held
    dpsgd.DPSGDRC([], C=1.0, sigma=0.0, norms=[a, junction.Junction(8)])


class Masked(torch.nn.Module):
    """A dropout and a frozen junction before a trained layer; ``seen`` has their outputs."""

    def __init__(self):
        super().__init__()
        self.drop, self.junction = junction.Dropout(0.4, site_id=2), junction.Junction(16, kind="rms", p=0.3, site_id=5)
        self.lin = torch.nn.Linear(16, 4, bias=False)

    def forward(self, x):
        d = self.drop(x)
        y, s = self.junction(d)
        self.seen = d.detach(), s.detach()
        return self.lin(y).square().mean((1, 2))


def test_every_mask_in_a_step_follows_its_key():
    # modules that the step was not told of: their masks are the step's, other ones every step
    model, x = Masked(), 1.0 + torch.rand(2, 5, 16)
    drv = dpsgd.DPSGDRC([model.lin], C=1.0, sigma=0.0, seed=3)
    masks = []
    for step in range(3):
        drv.steps = step
        drv.capture(lambda: model(x))
        key = dpsgd.step_seed(3, step)
        kept = [torch.from_numpy(J.dropout_factors(key, site, 10, 16, p)).view(2, 5, 16) != 0 for site, p in ((2, 0.4), (5, 0.3))]
        d, s = model.seen
        assert torch.equal(d != 0, kept[0]) and torch.equal(s != 0, kept[0] & kept[1])
        assert model.drop.seed == model.junction.seed == key
        masks.append(d != 0)
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])
    # a seed that the caller has set is left alone, unless the step was given the module
    model.drop.seed = 12345
    drv.capture(lambda: model(x))
    assert torch.equal(model.seen[0] != 0, torch.from_numpy(J.dropout_factors(12345, 2, 10, 16, 0.4)).view(2, 5, 16) != 0)
    assert model.drop.seed == 12345 and model.junction.seed == dpsgd.step_seed(3, 2)
    listed = dpsgd.DPSGDRC([model.lin], C=1.0, sigma=0.0, seed=4, dropouts=[model.drop])
    listed.capture(lambda: model(x))
    assert model.drop.seed == model.junction.seed == 4
    # and is the step's from then on, also in a step that was not given it
    drv.capture(lambda: model(x))
    assert model.drop.seed == dpsgd.step_seed(3, 2)
    # outside a step nothing changes it
    model.drop.seed = 0
    model(x)
    assert model.drop.seed == 0 and torch.equal(model.seen[0] != 0, torch.from_numpy(J.dropout_factors(0, 2, 10, 16, 0.4)).view(2, 5, 16) != 0)
    drv.remove_hooks(), listed.remove_hooks()


def test_a_step_keys_only_what_runs_in_it():
    # neither another thread's forward pass during the capture, nor any after one that failed
    import threading
    model, other, x = Masked(), Masked(), torch.rand(2, 5, 16)
    drv = dpsgd.DPSGDRC([model.lin], C=1.0, sigma=0.0, seed=3)

    def loss():
        t = threading.Thread(target=lambda: other(x))
        t.start()
        t.join()
        return model(x)
    drv.capture(loss)
    assert model.drop.seed == 3 and other.drop.seed == other.junction.seed == 0
    with pytest.raises(ZeroDivisionError):
        drv.capture(lambda: 1 / 0)
    other(x)
    assert other.drop.seed == 0
    drv.remove_hooks()


def test_backward_is_of_the_call_that_was_made():
    # the place and the kind are attributes: a caller may change them between a module's calls, and the
    # backward pass makes the masks of each call again
    x, t = torch.randn(2, 5, 16), torch.randn(2, 5, 16)
    drop, junc = junction.Dropout(0.4), junction.Junction(16, kind="rms", p=0.3)

    def outputs(ins):
        out = []
        for k, a in enumerate(ins):
            junc.site_id, junc.seed, junc.p, junc.kind = 3 + k, 40 + k, 0.3 + 0.2 * k, (dprc.RMSNORM, dprc.LAYERNORM)[k]
            drop.site_id, drop.seed, drop.p = 7 + k, 50 + k, 0.4 + 0.2 * k
            out.append(junc(drop(a))[0])
        return out
    one_by_one = []
    for k in range(2):
        ins = [x.clone().requires_grad_() for _ in range(2)]
        junc_out = outputs(ins[:k + 1])[k]
        one_by_one.append(torch.autograd.grad((junc_out * t).sum(), ins[k])[0])
    ins = [x.clone().requires_grad_() for _ in range(2)]
    both = torch.autograd.grad(sum((y * t).sum() for y in outputs(ins)), ins)
    for a, b in zip(both, one_by_one):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dual", ["x", "res", "weight", "bias"])
@pytest.mark.parametrize("grad", [True, False])
def test_forward_mode_is_refused(dual, grad):
    # there is no forward-mode rule: an output without its tangent would be taken for a constant
    import torch.autograd.forward_ad as fw
    t = dict(x=torch.randn(2, 5, 16), res=torch.randn(2, 5, 16), weight=torch.ones(16), bias=torch.zeros(16))
    junc, drop = junction.Junction(16), junction.Dropout(0.3)
    with fw.dual_level(), torch.set_grad_enabled(grad):
        t[dual] = fw.make_dual(t[dual], torch.ones_like(t[dual]))
        call = lambda: torch.func.functional_call(junc, {k: t[k] for k in ("weight", "bias")}, (t["x"], t["res"]))
        with pytest.raises((NotImplementedError, RuntimeError)):
            call()
        if dual in ("x", "res"):
            with pytest.raises((NotImplementedError, RuntimeError)):
                drop(t["x"], t["res"])
        plain = {k: fw.unpack_dual(v).primal for k, v in t.items()}
        y, _ = torch.func.functional_call(junc, {k: plain[k] for k in ("weight", "bias")}, (plain["x"], plain["res"]))
        assert fw.unpack_dual(y).tangent is None and drop(plain["x"], plain["res"]).shape == (2, 5, 16)


def test_micro_batches_take_keys_of_their_own():
    # rows are counted from 0 in every call, so captures under one key have the same masks; with another key they
    # have others, forwards and backwards
    model, x = Masked(), 1.0 + torch.rand(2, 5, 16)
    drv = dpsgd.DPSGDRC([model.lin], C=1.0, sigma=0.0, seed=3, norms=[model.junction])
    model.junction.p = 0.0
    E = []
    for key in (None, dpsgd.step_seed(3, 0), 99):
        _, pairs = drv.capture(lambda: model(x), **({} if key is None else dict(key=key)))
        used = dpsgd.step_seed(3, 0) if key is None else key
        assert model.drop.seed == model.junction.seed == used
        kept = torch.from_numpy(J.dropout_factors(used, 2, 10, 16, 0.4)).view(2, 5, 16) != 0
        assert torch.equal(model.seen[0] != 0, kept) and torch.equal(pairs[0][0] != 0, kept)
        E.append(pairs.vectors)
    assert torch.equal(E[0], E[1]) and not torch.equal(E[0], E[2])
    drv.remove_hooks()
