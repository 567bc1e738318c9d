"""Junctions in a model and in the private training step.

The Llama-shaped stack at small sizes with its residual sums, norms and dropout in
``junction.Junction``: its forward pass against the plain stack, its gradients against torch's
autograd of the plain formulas in 64 bits, and the step's norms, clipped sums and update of the
norms' parameters against the oracle on the tensors that the step captured.
"""

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import junction as J
from workloads import llama

pytestmark = pytest.mark.gpu

SIZES = dict(layers=2, hidden=128, mlp=256, heads=4, kv_heads=2, vocab=200)


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc, dpsgd, junction
    dprc.lib()
    return dprc, dpsgd, junction


def _model(dtype=torch.bfloat16, seed=1, **kw):
    return llama.build(seed=seed, device="cuda", dtype=dtype, **dict(SIZES, **kw))


def _tokens(B=3, T=40, seed=1):
    return llama.tokens(B, T, SIZES["vocab"], seed=seed, device="cuda")


def test_junctions_compute_the_plain_stack(mods):
    # same weights, rms norms, no dropout.  fp32: the two differ by the rounding of a few sums over
    # 128 columns per norm, through 5 norms
    plain, junc = _model(torch.float32), _model(torch.float32, junctions=True)
    junc.load_state_dict(plain.state_dict())
    tok = _tokens()
    a, b = plain(tok[:, :-1]), junc(tok[:, :-1])
    assert (a - b).abs().max() <= 1e-5 * a.abs().max()
    with torch.no_grad():
        assert torch.equal(junc(tok[:, :-1]), b)
    ga = torch.autograd.grad(llama.per_sample_loss(a, tok[:, 1:]).sum(), list(plain.parameters()))
    gb = torch.autograd.grad(llama.per_sample_loss(b, tok[:, 1:]).sum(), list(junc.parameters()))
    for (name, _), x, y in zip(plain.named_parameters(), ga, gb):
        assert (x - y).abs().max() <= 1e-4 * x.abs().max(), name


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_module_gradients(mods, kind):
    # fp32 against autograd of the formulas in 64 bits with the oracle's mask
    D, _, junction = mods
    B, T, n, p = 3, 21, 72, 0.25
    mod = junction.Junction(n, kind=kind, p=p, site_id=9).cuda()
    mod.seed = 77
    g = torch.Generator().manual_seed(3)
    x, res, ty, ts = (torch.randn(B, T, n, generator=g) for _ in range(4))
    with torch.no_grad():
        mod.weight.copy_(1 + 0.1 * torch.randn(n, generator=g))
        if mod.bias is not None:
            mod.bias.copy_(0.1 * torch.randn(n, generator=g))
    params = mod.parameters_in_order()
    for use in ("both", "y", "s"):
        ins = [t.cuda().requires_grad_() for t in (x, res)]
        y, s = mod(*ins)
        loss = sum((o * t.cuda()).sum() for o, t, k in ((y, ty, "y"), (s, ts, "s")) if use in ("both", k))
        got = torch.autograd.grad(loss, ins + params, allow_unused=True)
        f = torch.from_numpy(J.dropout_factors(77, 9, B * T, n, p)).view(B, T, n)
        ins64 = [t.double().requires_grad_() for t in (x, res)]
        par64 = [q.detach().cpu().double().requires_grad_() for q in params]
        s64 = ins64[1] + f * ins64[0]
        d = s64 - s64.mean(-1, keepdim=True) if kind == "layer" else s64
        y64 = d / torch.sqrt((d * d).mean(-1, keepdim=True) + float(np.float32(1e-5))) * par64[0]
        if len(par64) > 1:
            y64 = y64 + par64[1]
        loss64 = sum((o * t.double()).sum() for o, t, k in ((y64, ty, "y"), (s64, ts, "s")) if use in ("both", k))
        ref = torch.autograd.grad(loss64, ins64 + par64, allow_unused=True)
        for a, b in zip(got, ref):
            b = torch.zeros_like(a).cpu().double() if b is None else b
            # sums over 72 columns and 63 rows in fp32, a few roundings on top
            assert (a.cpu().double() - b).abs().max() <= 1e-5 * max(1.0, b.abs().max().item())
    mod.eval()
    y, s = mod(x.cuda(), res.cuda())
    assert torch.equal(s, x.cuda() + res.cuda())                      # no dropout outside training
    y, s = mod(x.cuda())
    assert torch.equal(s, x.cuda())


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_module_without_a_residual(mods, p):
    # as above, s handed on as the next residual; with p = 0 s is x itself
    D, _, junction = mods
    B, T, n = 2, 19, 72
    mod = junction.Junction(n, p=p, site_id=4).cuda()
    mod.seed = 5
    g = torch.Generator().manual_seed(4)
    x, ty, ts = (torch.randn(B, T, n, generator=g) for _ in range(3))
    f = torch.from_numpy(J.dropout_factors(5, 4, B * T, n, p)).view(B, T, n)
    x64 = x.double().requires_grad_()
    s64 = f * x64
    d = s64 - s64.mean(-1, keepdim=True)
    y64 = d / torch.sqrt((d * d).mean(-1, keepdim=True) + float(np.float32(1e-5)))
    ref = torch.autograd.grad((y64 * ty.double()).sum() + (s64 * ts.double()).sum(), x64)[0]
    xc = x.cuda().requires_grad_()
    y, s = mod(xc)
    got = torch.autograd.grad((y * ty.cuda()).sum() + (s * ts.cuda()).sum(), [xc, *mod.parameters()])
    assert (got[0].cpu().double() - ref).abs().max() <= 1e-5 * max(1.0, ref.abs().max().item())
    for q in mod.parameters():                                        # the weights alone, then neither
        assert torch.equal(torch.autograd.grad((mod(x.cuda())[0] * ty.cuda()).sum(), q)[0], got[1 if q is mod.weight else 2])
    for q in mod.parameters():
        q.requires_grad_(False)
    y2, s2 = mod(xc)
    alone = torch.autograd.grad((y2 * ty.cuda()).sum() + (s2 * ts.cuda()).sum(), xc)[0]
    assert torch.equal(alone, got[0]) and torch.equal(y2, y) and not mod(x.cuda())[0].requires_grad


def test_module_on_each_samples_last_token(mods):
    D, _, junction = mods
    mod = junction.Junction(80, kind="rms").cuda().eval()
    x, z = torch.randn(3, 7, 80, device="cuda"), torch.randn(3, 7, 80, device="cuda")
    with torch.no_grad():
        y, s = mod(x, z)
        for cut in (slice(-1, None), slice(2, 3), slice(2, 5)):
            y1, s1 = mod(x[:, cut], z[:, cut])
            assert torch.equal(y1, y[:, cut]) and torch.equal(s1, s[:, cut])


def test_step_trains_the_norms(mods):
    D, dpsgd, _ = mods
    C, sigma, k, lr, wd = 0.05, 0.6, 16, 1e-3, 0.01
    for norm, dropout, fused, estimator in (("rms", 0.0, True, "hutch"), ("layer", 0.1, True, "hutch"),
                                            ("layer", 0.1, False, "hutchpp")):
        model = _model(junctions=True, norm=norm, dropout=dropout)
        tok = _tokens()
        drv = dpsgd.DPSGDRC(model.linears(), C=C, sigma=sigma, k=k, s=4, r=8, estimator=estimator, seed=11, lr=lr,
                            weight_decay=wd, fused_adamw=fused, norms=model.norms())
        N = drv.vec_master.shape[1]
        assert N == 5 * 128 * (2 if norm == "layer" else 1)
        loss_fn = lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:])
        losses, pairs = drv.capture(loss_fn)
        key = dpsgd.step_seed(11, 0)
        G = drv._G.clone()
        assert G.shape == (3, N) and torch.isfinite(G).all() and (G.abs().sum(1) > 0).all()
        n2, c, grads = drv.private_grads(pairs, key, noise=not fused)
        torch.cuda.synchronize()
        G64 = est.as_f64(G)
        lin = [(est.hutch_layer(est.as_f64(A), est.as_f64(E), k, key, j) if estimator == "hutch" else
                est.hutchpp_layer(est.as_f64(A), est.as_f64(E), 4, 8, key, j)) for (A, E, j) in pairs]
        ref = J.norm_vectors(G64) + sum(lin)
        assert np.all(np.abs(n2.cpu().numpy() - ref) <= 1e-3 * ref)
        assert np.all(J.norm_vectors(G64) > 0.0)
        c_ref = est.clip_scale(n2.cpu().numpy().astype(np.float64), C)
        assert np.allclose(c.cpu().numpy(), c_ref, rtol=1e-6)
        clipped = J.clip_accumulate_vectors(G64, c_ref)
        nl = len(model.linears())
        assert len(grads) == nl + 1 and grads[nl].shape == (1, N)
        noisy = est.add_noise(clipped[None], sigma, C, key, nl)
        want = clipped[None] if fused else noisy
        assert np.max(np.abs(est.as_f64(grads[nl]) - want)) <= 1e-5 * np.max(np.abs(want))
        master0 = est.as_f64(drv.vec_master)
        (drv.update if fused else drv.apply)(grads, *((3, key) if fused else (3,)))
        torch.cuda.synchronize()
        th, _, _ = est.adamw(master0, noisy / 3, 0.0, 0.0, 1, lr, 0.9, 0.999, 1e-8, 0.0)     # no decay
        firm = np.abs(noisy / 3) > 1e-5
        got = est.as_f64(drv.vec_master)
        assert firm.mean() > 0.99 and np.max(np.abs(got - th)[firm]) <= 1e-6 and np.max(np.abs(got - th)) <= 2.1e-3
        # the modules' parameters are what was updated
        flat = torch.cat([q.detach().view(-1) for m in model.norms() for q in m.parameters_in_order()])
        assert torch.equal(flat, drv.vec_master[0].bfloat16())
        drv.remove_hooks()


def test_captured_norm_gradients_are_each_samples_own(mods):
    # fp32 without dropout: sample i alone through torch's autograd of the plain stack gives row i
    D, dpsgd, _ = mods
    plain, model = _model(torch.float32), _model(torch.float32, junctions=True)
    model.load_state_dict(plain.state_dict())
    tok = _tokens()
    drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, norms=model.norms())
    drv.capture(lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]))
    for i in range(3):
        li = llama.per_sample_loss(plain(tok[i:i + 1, :-1]), tok[i:i + 1, 1:])[0]
        ref = torch.cat(torch.autograd.grad(li, [m.weight for m in plain.norms()]))
        assert (drv._G[i] - ref).abs().max() <= 1e-4 * ref.abs().max(), i
    # outside a step the modules give ordinary gradients, as often as wanted
    assert all(m.sink is None for m in model.norms())
    for _ in range(2):
        gw = torch.autograd.grad(llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]).sum(), [m.weight for m in model.norms()])
        ref = drv._G.sum(0)
        assert (torch.cat(gw) - ref).abs().max() <= 1e-5 * ref.abs().max()
    drv.remove_hooks()


def test_dropout_is_fresh_every_step_and_training_stays_finite(mods):
    D, dpsgd, _ = mods
    model = _model(junctions=True, norm="layer", dropout=0.2)
    tok = _tokens()
    drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.5, k=16, seed=2, lr=1e-3, norms=model.norms())
    w0 = drv.vec_w.clone()
    seeds = set()
    for _ in range(3):
        losses = drv.step(lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]))
        assert torch.isfinite(losses).all() and torch.isfinite(drv.last["n2"]).all() and (drv.last["c"] > 0).all()
        seeds.add(model.norms()[0].seed)
    assert len(seeds) == 3 and len({m.site_id for m in model.norms()}) == 5
    assert not torch.equal(drv.vec_w, w0)
    drv.remove_hooks()


def test_norms_that_a_step_cannot_train_are_refused(mods):
    D, dpsgd, junction = mods
    model = _model(junctions=True)
    tok = _tokens()
    with pytest.raises(ValueError):                                   # parameters of two dtypes
        dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, norms=[model.norm, junction.Junction(8).cuda()])
    unused = junction.Junction(128, kind="rms").cuda().bfloat16()
    drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, norms=model.norms() + [unused])
    with pytest.raises(RuntimeError):
        drv.capture(lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]))
    drv.remove_hooks()
    model = _model(junctions=True)
    drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, norms=model.norms())
    with pytest.raises(RuntimeError):                                 # twice in one step
        drv.capture(lambda: llama.per_sample_loss(model(tok[:, :-1]) + model(tok[:, :-1]), tok[:, 1:]))
    drv.remove_hooks()


@pytest.mark.parametrize("res", [False, True])
def test_dropout_module(mods, res):
    # outputs and gradients are the mask's factors, bit for bit in fp32 (one product, one sum)
    D, _, junction = mods
    B, T, n, p = 3, 17, 75, 0.3
    mod = junction.Dropout(p, site_id=6)
    mod.seed = 31
    x, z, t = (torch.randn(B, T, n, device="cuda") for _ in range(3))
    f = torch.from_numpy(J.dropout_factors(31, 6, B * T, n, p)).view(B, T, n).float().cuda()
    ins = [x.clone().requires_grad_()] + ([z.clone().requires_grad_()] if res else [])
    y = mod(*ins)
    want = torch.addcmul(z.double(), f.double(), x.double()) if res else (f * x).double()
    assert (y.double() - want).abs().max() <= 2.0 ** -24 * 2 * ((f * x).abs().max() + want.abs().max())
    grads = torch.autograd.grad((y * t).sum(), ins)
    assert torch.equal(grads[0], f * t) and (not res or torch.equal(grads[1], t))
    spread = torch.autograd.grad(mod(*ins).sum(), ins)                # a gradient without strides of its own
    assert torch.equal(spread[0], f) and (not res or torch.equal(spread[1], torch.ones_like(z)))
    part = mod(x[:, :1], *([z[:, :1]] if res else []))
    assert not part.requires_grad and part.shape == (B, 1, n)
    mod.eval()
    assert mod(x) is x and torch.equal(mod(x, z), x + z)
    with torch.no_grad():
        assert torch.equal(mod(x, z), x + z)


def test_step_keys_the_dropouts(mods):
    # what a step captures as input of the layer after a dropout is zero exactly where that step's mask is
    D, dpsgd, _ = mods
    p = 0.25
    model = _model(junctions=True, dropout=p)
    tok = _tokens()
    drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, seed=4, norms=model.norms(), dropouts=model.dropouts())
    sites = [m.site_id for m in model.norms() + model.dropouts()]
    assert len(set(sites)) == len(sites)
    seen = []
    for _ in range(2):
        seen_now = []
        hooks = [b.down.register_forward_hook(lambda m, i, o: seen_now.append(i[0].detach())) for b in model.blocks]
        drv.step(lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:]))
        for h in hooks:
            h.remove()
        assert len({m.seed for m in model.norms() + model.dropouts()}) == 1
        for a, m in zip(seen_now, model.dropouts()):
            B, T, n = a.shape
            f = torch.from_numpy(J.dropout_factors(m.seed, m.site_id, B * T, n, p)).view(B, T, n)
            assert (a.cpu()[f == 0] == 0).all() and (a.cpu()[f != 0] != 0).float().mean() > 0.99
        seen.append((model.dropouts()[0].seed, seen_now))
    assert seen[0][0] != seen[1][0]
    drv.remove_hooks()
