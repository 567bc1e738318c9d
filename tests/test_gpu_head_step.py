"""The head, rotary positions and the joint clipping in a model and in the private training step."""

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import head as O
from workloads import llama

pytestmark = pytest.mark.gpu

SIZES = dict(layers=2, hidden=128, mlp=256, heads=4, kv_heads=2, vocab=9000)
U = 2.0 ** -24
f64 = est.as_f64


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc, dpsgd, head, rotary
    dprc.lib()
    return dprc, dpsgd, head, rotary


def _model(dtype=torch.bfloat16, seed=1, **kw):
    return llama.build(seed=seed, device="cuda", dtype=dtype, **dict(SIZES, **kw))


def _tokens(B=3, T=40, seed=1):
    return llama.tokens(B, T, SIZES["vocab"], seed=seed, device="cuda")


def _loss(model, tok):
    return lambda: model(tok[:, :-1], tok[:, 1:]).mean(dim=1)


def test_they_compute_the_plain_stack(mods):
    # fp32: sums of 128 to 9000 terms in other orders, through two blocks
    plain, own = _model(torch.float32), _model(torch.float32, head=True, rotary=True)
    own.load_state_dict(plain.state_dict())
    tok = _tokens()
    a, b = llama.per_sample_loss(plain(tok[:, :-1]), tok[:, 1:]), _loss(own, tok)()
    assert (a - b).abs().max() <= 1e-5 * a.abs().max()
    with torch.no_grad():
        assert torch.equal(_loss(own, tok)(), b)
    ga = torch.autograd.grad(a.sum(), list(plain.parameters()))
    gb = torch.autograd.grad(b.sum(), list(own.parameters()))
    for (name, _), x, y in zip(plain.named_parameters(), ga, gb):
        assert (x - y).abs().max() <= 1e-4 * x.abs().max(), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_head_module_gradients(mods, dtype):
    _, _, head, _ = mods
    lin = torch.nn.Linear(72, 1111, bias=False, device="cuda", dtype=dtype)
    mod = head.Head(lin)
    g = torch.Generator().manual_seed(3)
    h = torch.randn(2, 21, 72, generator=g).to(dtype).cuda().requires_grad_()
    y = torch.randint(0, 1111, (2, 21), generator=g).cuda()
    y[0, 3:9] = -100
    w = torch.randn(2, 21, generator=g).cuda()
    loss = mod(h, y)
    got = torch.autograd.grad((loss * w).sum(), [h, lin.weight])
    hn, Wn, yn = f64(h.detach()), f64(lin.weight.detach()), y.cpu().numpy()
    rl, rz = O.loss(hn, Wn, yn)
    assert np.abs(f64(loss.detach()) - rl).max() <= 200 * U * (1 + np.abs(rz).max())
    E = O.errors(hn, Wn, yn, rz, f64(w))
    # E, then the sum, are rounded to the type: 2 r of the terms' magnitudes; fp32: chains of 1111 and 42 sums
    r = 2 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    for a, ref, mag in ((got[0], E @ Wn, np.abs(E) @ np.abs(Wn)),
                        (got[1], np.einsum("btv,btd->vd", E, hn), np.einsum("btv,btd->vd", np.abs(E), np.abs(hn)))):
        assert (np.abs(f64(a) - ref) <= (r + 1300 * U) * mag + 1e-30).all()
    assert a.dtype == dtype
    # either gradient alone, none, and strided hidden states
    alone = torch.autograd.grad((mod(h, y) * w).sum(), h)[0]
    assert torch.equal(alone, got[0])
    assert torch.equal(torch.autograd.grad((mod(h.detach(), y) * w).sum(), lin.weight)[0], got[1])
    wide = torch.zeros(2, 21, 80, device="cuda", dtype=dtype)
    wide[..., :72] = h.detach()
    assert torch.equal(mod(wide[..., :72], y).detach(), loss.detach())
    assert torch.equal(mod(h.detach().transpose(0, 1).contiguous().transpose(0, 1), y).detach(), loss.detach())
    with torch.no_grad():
        assert torch.equal(mod(h, y), loss.detach()) and not mod(h, y).requires_grad


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rotary_module_gradients(mods, dtype):
    _, _, _, rotary = mods
    rot = rotary.Rotary(64, dim=48, interleaved=True, scaling=dict(kind="ramp", factor=8, original=256))
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn(2, 9, h, 64, generator=g).to(dtype).cuda().requires_grad_() for h in (4, 2))
    pos = torch.randint(0, 2000, (2, 9), generator=g)
    a, b = rot(q, k, pos=pos.cuda(), out_dtype=torch.float32, heads_first=True)
    ga, gb = torch.randn(a.shape, generator=g).cuda(), torch.randn(b.shape, generator=g).cuda()
    gq, gk = torch.autograd.grad((a * ga).sum() + (b * gb).sum(), [q, k])
    assert gq.dtype == dtype and a.dtype == torch.float32 and a.stride(1) == 64
    f = rot.freqs.numpy()
    r = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    for x, y, gx, gy in ((q, a, gq, ga), (k, b, gk, gb)):
        ref = O.rotary(f64(x.detach()), f, pos.numpy(), rot.scale, True)
        assert np.abs(f64(y.detach()) - ref).max() <= 40 * U * np.abs(ref).max()
        ref = O.rotary(f64(gy), f, pos.numpy(), rot.scale, True, True)
        assert (np.abs(f64(gx) - ref) <= 40 * U * np.abs(ref).max() + r * np.abs(ref)).all()
    # a gradient that is not laid out as heads (a broadcast one), and one result unused
    gq2, gk2 = torch.autograd.grad(rot(q, k, pos=pos.cuda())[0].float().sum(), [q, k])
    ref = O.rotary(np.ones(q.shape), f, pos.numpy(), rot.scale, True, True)
    assert (np.abs(f64(gq2) - ref) <= 40 * U + r * np.abs(ref)).all() and not gk2.any()
    one = rot(q.detach()[:, -1:], start=8)                   # a single token of a longer run
    whole = rot(q.detach())
    assert torch.equal(one, whole[:, -1:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_modules_of_broadcast_inputs(mods, dtype):
    """One sample's hidden states and one head's features for all: gradients are the sums over what shares them."""
    _, _, head, rotary = mods
    g = torch.Generator().manual_seed(9)
    mod = head.Head(torch.nn.Linear(40, 300, bias=False, device="cuda", dtype=dtype))
    h = torch.randn(1, 13, 40, generator=g).to(dtype).cuda().requires_grad_()
    y = torch.randint(0, 300, (3, 13), generator=g).cuda()
    whole = h.detach().expand(3, 13, 40).contiguous().requires_grad_()
    assert torch.equal(mod(h.expand(3, 13, 40), y), mod(whole, y))
    a, = torch.autograd.grad(mod(h.expand(3, 13, 40), y).mean(), h)      # a broadcast gradient of the losses, too
    b, = torch.autograd.grad(mod(whole, y).mean(), whole)
    assert torch.equal(a, b.sum(0, keepdim=True))
    rot = rotary.Rotary(20, dim=12)
    k = torch.randn(2, 9, 1, 20, generator=g).to(dtype).cuda().requires_grad_()
    w = torch.randn(2, 9, 5, 20, generator=g).to(dtype).cuda()
    each = k.detach().expand(2, 9, 5, 20).contiguous().requires_grad_()
    assert torch.equal(rot(k.expand(2, 9, 5, 20)), rot(each))
    a, = torch.autograd.grad((rot(k.expand(2, 9, 5, 20)) * w).sum(), k)
    b, = torch.autograd.grad((rot(each) * w).sum(), each)
    assert torch.equal(a, b.sum(2, keepdim=True))


def test_private_step_with_a_head(mods):
    """Estimates and clipped sums of the head against those of its stored gradient, and the update of its weight."""
    D, dpsgd, _, _ = mods
    model, tok = _model(head=True, rotary=True, junctions=True), _tokens()
    drv = dpsgd.DPSGDRC(model.linears(), C=0.7, sigma=0.5, k=16, lr=1e-2, norms=model.norms(), head=model.head, seed=5)
    losses, pairs = drv.capture(_loss(model, tok))
    key, part, nl = dpsgd.step_seed(5, 0), pairs.head, len(drv.linears)
    W = model.lm_head.weight.detach()
    E = D.dprc_head_errors(part.h, W, part.target, part.lse, part.g)
    ref = D.dprc_head_loss(part.h, W, part.target)[0].mean(1)
    assert torch.equal(losses, ref)
    own = sum(est.hutch_layer(f64(part.h), f64(E[..., v:v + D.HEAD_BLOCK]), 16, key, nl + b)
              for b, v in enumerate(range(0, SIZES["vocab"], D.HEAD_BLOCK)))
    n2, c, grads = drv.private_grads(pairs, key, noise=False)
    rest = dpsgd.Pairs(pairs, pairs.vectors)
    drv.head = None
    others, _ = drv.estimate(rest, key)
    drv.head = model.head
    np.testing.assert_allclose(f64(n2), f64(others) + own, rtol=1e-3)
    assert len(grads) == nl + 2 and grads[-1].shape == (128, SIZES["vocab"])
    rg = est.clip_accumulate(f64(part.h), f64(E), f64(c))
    assert np.linalg.norm(f64(grads[-1]) - rg) <= 1e-5 * np.linalg.norm(rg)
    # the same step through the fused update
    before, master = W.clone(), drv.head_master.clone()
    drv.step(_loss(model, tok))
    want = est.add_noise(f64(grads[-1]), 0.5, 0.7, key, nl + 1) / 3
    moved = f64(master - drv.head_master)
    big = np.abs(want) > 1e-6
    np.testing.assert_allclose(moved[big], (1e-2 * want / (np.abs(want) + 1e-8))[big], rtol=1e-3)
    assert torch.equal(model.lm_head.weight, drv.head_master.t().to(torch.bfloat16)) and not torch.equal(before, W)
    drv.remove_hooks()


@pytest.mark.parametrize("fused", [True, False])
def test_clipped_updates(mods, fused):
    D, dpsgd, _, _ = mods
    tok = _tokens()
    kw = dict(C=0.7, sigma=0.5, k=16, lr=1e-2, seed=5, fused_adamw=fused)
    model = _model(head=True, rotary=True)
    drv = dpsgd.DPSGDRC(model.linears(), head=model.head, max_norm=0.01, **kw)
    noisy = drv.private_grads(drv.capture(_loss(model, tok))[1], dpsgd.step_seed(5, 0))[2]
    ref, norm = O.clip([f64(g) / 3 for g in noisy], 0.01)
    before = [m.clone() for m in drv._masters()]
    drv.step(_loss(model, tok))
    np.testing.assert_allclose(f64(drv.last["norm"]), norm, rtol=1e-6)
    for b, m, g in zip(before, drv._masters(), ref):
        want, moved = 1e-2 * g / (np.abs(g) + 1e-8), f64(b - m)
        # a master near 0.02 moves by 0.01: its own rounding is 2 u 0.03; eps is above most of what is left of g
        assert (np.abs(moved - want) <= 4 * U * 0.1 + 1e-3 * np.abs(want)).all()
    drv.remove_hooks()


def test_they_train_together(mods):
    """Rotary positions, junctions, the head and the clipping in one run: a few steps without noise on one batch."""
    D, dpsgd, _, _ = mods
    model, tok = _model(head=True, rotary=True, junctions=True, norm="layer", dropout=0.1), _tokens()
    drv = dpsgd.DPSGDRC(model.linears(), C=10.0, sigma=0.0, k=16, lr=1e-3, norms=model.norms(), head=model.head,
                        dropouts=model.dropouts(), max_norm=1.0)
    seen = []
    for _ in range(4):
        losses = drv.step(_loss(model, tok))
        assert losses.isfinite().all() and drv.last["n2"].isfinite().all() and drv.last["norm"].isfinite().all()
        seen.append(drv.last["n2"].clone())
    assert not torch.equal(seen[0], seen[1]) and all(w.isfinite().all() for w in model.parameters())
    drv.remove_hooks()


def test_rotary_first_called_for_inference(mods):
    rot = mods[3].Rotary(8)
    x = torch.randn(2, 3, 4, 8, device="cuda", requires_grad=True)
    with torch.inference_mode():
        y = rot(x)
    g, = torch.autograd.grad(rot(x).sum(), x)            # the frequencies are saved for this
    assert torch.equal(rot(x.detach()), y) and g.isfinite().all()


def test_a_captured_pass(mods):
    """Losses and gradients of the model in a graph, replayed on other tokens."""
    model = _model(head=True, rotary=True)
    params = list(model.parameters())
    tok = _tokens()

    def run():
        losses = _loss(model, tok)()
        return [losses.detach(), *torch.autograd.grad(losses.sum(), params)]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for seed in (1, 2, 3):
        tok.copy_(_tokens(seed=seed))
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        want = run()
        assert torch.equal(got[0], want[0])
        # the embedding's gradient adds with atomics
        for (name, _), a, b in zip(model.named_parameters(), got[1:], want[1:]):
            assert torch.equal(a, b) or (name == "embed.weight" and (a - b).abs().max() <= 0.02 * b.abs().max()), name


def test_launches_are_traced(mods):
    from test_gpu_trace import _trace
    D = mods[0]
    bf = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    tokens = lambda T, V: torch.randint(0, V, (1, T), device="cuda")
    ones = lambda T: torch.ones(1, T, device="cuda")
    small, large = torch.randn(100, device="cuda"), torch.randn(100000, device="cuda")

    def back(T, d, V, **kw):
        h, W, y = bf(1, T, d), bf(V, d) * 0.1, tokens(T, V)
        lse = D.dprc_head_loss(h, W, y)[1]
        return lambda: D.dprc_head_backward(h, W, y, lse, ones(T), **kw)
    for call, kinds in (
            (lambda: D.dprc_head_loss(bf(1, 9, 64), bf(300, 64), tokens(9, 300)), ["head_sums", "head_join"]),
            (lambda: D.dprc_head_loss(bf(1, 9, 65), bf(300, 65), tokens(9, 300)), ["head_rows", "head_sums", "head_join"]),
            (back(40, 64, 500, hidden_grad=False), ["head_rows", "head_errors", "head_weight"]),
            (back(40, 64, 200, weight_grad=False), ["head_rows", "head_errors", "head_back"]),
            (back(40, 64, 200), ["head_rows", "head_errors", "head_back"]),                        # one launch for both
            (back(40, 64, 50000), ["head_rows", "head_errors", "head_back", "head_weight", "head_rows"]),
            (lambda: D.dprc_rotary([bf(1, 5, 2, 8), bf(1, 5, 1, 8)], torch.ones(4, dtype=torch.float64, device="cuda")), ["rotary"]),
            (lambda: D.dprc_grad_clip([small], 1.0), ["grad_scale"]),
            (lambda: D.dprc_grad_clip([large, small], 1.0), ["grad_squares", "grad_scale"]),
            (lambda: D.dprc_grad_norm([small]), ["grad_squares", "grad_squares"])):
        names, ms = _trace(D, call)
        assert names == kinds and all(0 < m < 1000 for m in ms), (names, kinds)
