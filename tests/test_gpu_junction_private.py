"""The norms' part in a private step's estimates, the masks of modules that a step was not given, and
the junction's gradient in bf16, on the GPU.

u = 2^-24 and r = 2^-8 are the roundings to fp32 and bf16.
"""

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import junction as J
from oracle.estimators import as_f64
from workloads import llama

pytestmark = pytest.mark.gpu

U, R = 2.0 ** -24, 2.0 ** -8
SIZES = dict(layers=2, hidden=128, mlp=256, heads=4, kv_heads=2, vocab=200)


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc, dpsgd, junction
    dprc.lib()
    return dprc, dpsgd, junction


def _stack(**kw):
    return llama.build(seed=1, device="cuda", **dict(SIZES, junctions=True, **kw))


def _loss(model, tok):
    return lambda: llama.per_sample_loss(model(tok[:, :-1]), tok[:, 1:])


def _tokens(B=3, T=40, seed=1):
    return llama.tokens(B, T, SIZES["vocab"], seed=seed, device="cuda")


@pytest.mark.parametrize("estimator", ["hutch", "hutchpp"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_estimates_hold_the_norms_part(mods, norm, estimator):
    # Beside the linear layers' the norms' squared gradients are small (3e-4 of n2 here), so they are looked for in
    # the difference that they make: the same pairs and key with and without them.  Each side is a sum of one
    # term a layer, every partial sum rounded once: 2 (layers + 2) u of n2.
    D, dpsgd, _ = mods
    model, key = _stack(norm=norm), 77
    drv = dpsgd.DPSGDRC(model.linears(), C=0.05, sigma=0.0, k=16, s=4, r=8, estimator=estimator, norms=model.norms())
    _, pairs = drv.capture(_loss(model, _tokens()))
    linear = D.dprc_norm_hutch(pairs, 16, key) if estimator == "hutch" else D.dprc_norm_hutchpp(pairs, 4, 8, key)
    linear = as_f64(linear)
    for factor in (1.0, 100.0):                                        # as they are, and as most of n2
        pairs.vectors.mul_(factor)
        part = J.norm_vectors(pairs.vectors)
        n2, c = drv.estimate(pairs, key)
        tol = 2 * (len(pairs) + 2) * U * (linear + part)
        assert np.all(part > 20 * tol) and (factor == 1.0 or np.all(part > linear))
        assert np.all(np.abs(as_f64(n2) - linear - part) <= tol)
        assert np.allclose(as_f64(c), est.clip_scale(linear + part, 0.05), rtol=1e-5)
    drv.remove_hooks()


def test_captures_do_not_mix(mods):
    D, dpsgd, _ = mods
    model = _stack(norm="layer")
    drv = dpsgd.DPSGDRC(model.linears(), C=0.05, sigma=0.0, k=16, norms=model.norms())
    toks = _tokens(3, seed=1), _tokens(2, seed=2)
    alone = [drv.private_grads(drv.capture(_loss(model, t))[1], 5) for t in toks]
    both = [drv.capture(_loss(model, t))[1] for t in toks]
    for use in (0, 1, 0):
        n2, c, grads = drv.private_grads(both[use], 5)
        for a, b in zip((n2, c, *grads), (*alone[use][:2], *alone[use][2])):
            assert torch.equal(a, b)
    with pytest.raises(ValueError):
        drv.private_grads(list(both[0]), 5)
    drv.remove_hooks()


def test_masks_of_modules_that_the_step_was_not_given(mods):
    # norms= alone: the MLP's dropouts run under the step's key too, and so do junctions when nothing is listed
    D, dpsgd, _ = mods
    p = 0.25
    for listed in (True, False):
        model, tok = _stack(dropout=p), _tokens()
        drv = dpsgd.DPSGDRC(model.linears(), C=1.0, sigma=0.0, seed=4, norms=model.norms() if listed else ())
        seen, sums = [], []
        hooks = [model.blocks[1].down.register_forward_hook(lambda m, i, o: seen.append(i[0].detach())),
                 model.blocks[0].norm1.register_forward_hook(lambda m, i, o: sums.append(o[1].detach()))]
        for step in range(2):
            key = dpsgd.step_seed(4, step)
            drv.step(_loss(model, tok))
            for a, m in ((seen[-1], model.blocks[1].act_drop), (sums[-1], model.blocks[0].norm1)):
                B, T, n = a.shape
                dropped = torch.from_numpy(J.dropout_factors(key, m.site_id, B * T, n, p) == 0).view(B, T, n).cuda()
                assert m.seed == key and (a[dropped] == 0).all() and (a[~dropped] != 0).float().mean() > 0.99
        assert not torch.equal(seen[0] == 0, seen[1] == 0)
        for h in hooks:
            h.remove()
        drv.remove_hooks()


def test_norm_over_its_input(mods):
    # y in x's place: s is kept apart, and the gradient is that of the call with y elsewhere
    D, _, _ = mods
    for dtype, n in ((torch.bfloat16, 200), (torch.float32, 75)):
        x, w = torch.randn(3, 17, n, device="cuda").to(dtype), torch.randn(n, device="cuda").to(dtype)
        y, s, mean, rstd = D.dprc_layernorm(x, w)
        a = x.clone()
        y1, s1, m1, r1 = D.dprc_layernorm(a, w, y=a)
        assert y1 is a and torch.equal(y1, y) and torch.equal(s1, x) and torch.equal(m1, mean) and torch.equal(r1, rstd)
        for u, v in zip(D.dprc_layernorm_backward(y, s, w, mean, rstd), D.dprc_layernorm_backward(y, s1, w, m1, r1)):
            assert (u is None and v is None) or torch.equal(u, v)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("shift", [0.0, 4.0, 64.0])
def test_module_gradients_in_bf16(mods, kind, shift):
    """Against the gradient of the forward pass in 64 bits, at the sum as it is before it is rounded.

    The backward pass has that sum rounded to bf16, so xh is off by at most h = r |s| rstd (and the few u of
    fp32 arithmetic, which 2^-12 of everything covers here): beside a residual far from zero, with a small
    spread, that is far more than the rounding of the outputs.  dx is rstd (g - mean(g) - xh mean(g xh)) and
    moves by rstd (h |mean(g xh)| + (|xh| + h) mean(|g| h)), dw by the sum of |dy| h.  The gradients of weight
    and bias are rounded to bf16 at the end, dx and dh too."""
    D, _, junction = mods
    B, T, n, p = 2, 30, 136, 0.2
    mod = junction.Junction(n, kind=kind, p=p, site_id=3).cuda().bfloat16()
    mod.seed = 9
    g = torch.Generator().manual_seed(5)
    x, res, dy, ds = (torch.randn(B, T, n, generator=g).bfloat16() for _ in range(4))
    res = (res.float() + shift).bfloat16()
    with torch.no_grad():
        mod.weight.copy_(1 + 0.1 * torch.randn(n, generator=g))
        if mod.bias is not None:
            mod.bias.copy_(0.1 * torch.randn(n, generator=g))
    ins = [t.cuda().requires_grad_() for t in (x, res)]
    y, s = mod(*ins)
    got = torch.autograd.grad((y.float() * dy.cuda().float()).sum() + (s.float() * ds.cuda().float()).sum(),
                              ins + mod.parameters_in_order())
    s64 = J.dropout(x, 9, 3, p, res=res)
    w64, dy64, ds64 = as_f64(mod.weight), as_f64(dy), as_f64(ds)
    _, mean, rstd = J.norm(s64, eps=1e-5, rms=kind == "rms")
    dx, dw, db = J.norm_backward(dy64, s64, w64, mean, rstd, ds=ds64)
    r3 = rstd.reshape(B, T, 1)
    xh = (s64 - (0.0 if mean is None else mean.reshape(B, T, 1))) * r3
    gg = dy64 * w64
    h = R * np.abs(s64) * r3
    off = r3 * (h * np.abs((gg * xh).mean(-1, keepdims=True)) + (np.abs(xh) + h) * (np.abs(gg) * h).mean(-1, keepdims=True))
    small = r3 * (np.abs(gg) + np.abs(gg).mean(-1, keepdims=True) + np.abs(xh) * np.abs(gg * xh).mean(-1, keepdims=True))
    tol = off + 2.0 ** -12 * (small + np.abs(ds64)) + R * np.abs(dx) + R * off
    f = J.dropout_factors(9, 3, B * T, n, p).reshape(B, T, n)
    assert np.all(np.abs(as_f64(got[1]) - dx) <= tol)
    assert np.all(np.abs(as_f64(got[0]) - f * dx) <= f * tol * (1 + R))
    dwo = (np.abs(dy64) * h).sum(1)
    for grad, ref, o, mag in ((got[2], dw, dwo, np.abs(dy64 * xh).sum(1)), (got[3] if len(got) > 3 else None, db, 0.0 * dwo, np.abs(dy64).sum(1))):
        if grad is not None:
            ref, o, mag = ref.sum(0), o.sum(0), mag.sum(0)
            assert np.all(np.abs(as_f64(grad) - ref) <= o * (1 + R) + 2.0 ** -12 * mag + R * np.abs(ref))


def test_gradients_of_rows_past_32_bit_elements(mods):
    """More than 2^32 elements: every part of dw and db counts.

    2^27 + 5 rows of 40 in bf16 are dealt to 768 workgroups, 32 rows a round: 5462 rounds each.  A column's chain is
    those, 3 sums over lanes, 3 over waves, then 48 parts and 16 groups: under 5600 roundings.  The terms are off by 4 u
    each (xh; 8 allowed).  A part that were lost, or counted twice, is 1 / 768 of the sums, whose terms hardly
    cancel: half of the rows are the others' negatives, and dy follows s about a mean of its own."""
    D, _, _ = mods
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB of free memory")
    rows, n = (1 << 27) + 5, 40
    g = torch.Generator().manual_seed(2)
    base = torch.randn(32, n, generator=g).bfloat16()
    base = torch.cat([base, -base])
    grad = (3.0 * base.float() + 3.0).bfloat16()
    _, m64, r64 = J.norm(base.view(1, 64, n))
    m32, r32 = torch.from_numpy(m64).float(), torch.from_numpy(r64).float()
    tile = lambda t: t.cuda().repeat((rows + 63) // 64, *(1,) * (t.dim() - 1))[:rows]
    dx, _, dw, db = D.dprc_layernorm_backward(tile(grad).view(1, rows, n), tile(base).view(1, rows, n), None, tile(m32), tile(r32))
    del dx
    xh = (as_f64(base) - as_f64(m32)[:, None]) * as_f64(r32)[:, None]
    full, tail = rows // 64, rows % 64
    for got, terms in ((dw, as_f64(grad) * xh), (db, as_f64(grad))):
        want, mag = (full * t.sum(0) + t[:tail].sum(0) for t in (terms, np.abs(terms)))
        tol = (5600 + 8) * U * mag
        assert np.all(np.abs(want) / 768 > 1.5 * tol)
        assert np.all(np.abs(as_f64(got)[0] - want) <= tol)
