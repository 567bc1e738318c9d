"""Refusals of the output head, rotary positions and the joint norm, by the library (pointers that are never
followed) and by the binding (a library that only records its calls)."""

import ctypes
import math
import os
import types

import numpy as np
import pytest
import torch

from oracle import head as O
from paper_2605_24879_amd import dprc

built = pytest.mark.skipif(not os.path.exists(dprc.LIB_PATH), reason="libdprc.so not built")
INVALID, UNSUPPORTED, SMALL = 1, 2, 3
PTR = 0x100000


def head(**kw):
    f = dict(h=PTR, W=2 * PTR, target=3 * PTR, B=2, T=8, d=64, V=300, ldh=64, ldw=64, dtype=dprc.BF16, piece=0)
    f.update(kw)
    return dprc.HEAD.pack(*f.values())


def norms(**kw):
    f = dict(k=4, probe=0, seed=0, side=0, layer_id=0, n2=9 * PTR, accumulate=0)
    f.update(kw)
    return dprc.HEAD_NORMS.pack(*f.values())


BIG = 1 << 50


def loss(H, loss=4 * PTR, lse=5 * PTR, ws=PTR, n=BIG):
    return dprc.lib().dprc_head_loss(H, loss, lse, ws, n, None)


def errors(H, lse=4 * PTR, g=5 * PTR, v0=0, nv=10, E=6 * PTR, lde=10, ws=PTR, n=BIG):
    return dprc.lib().dprc_head_errors(H, lse, g, v0, nv, E, lde, ws, n, None)


def back(H, lse=4 * PTR, g=5 * PTR, dh=6 * PTR, lddh=64, dW=7 * PTR, lddw=64, nm=None, ws=PTR, n=BIG):
    return dprc.lib().dprc_head_backward(H, lse, g, dh, lddh, dW, lddw, nm, ws, n, None)


def clip(H, lse=4 * PTR, g=5 * PTR, c=6 * PTR, grad=7 * PTR, ldg=300, ws=PTR, n=BIG):
    return dprc.lib().dprc_head_clip_accumulate(H, lse, g, c, grad, ldg, 0, ws, n, None)


@built
@pytest.mark.parametrize("call", [loss, errors, back, clip])
def test_head_descriptions(call):
    for bad in (dict(h=0), dict(W=0), dict(target=0), dict(B=0), dict(T=-1), dict(d=0), dict(V=0), dict(ldh=63), dict(ldw=63),
                dict(dtype=2), dict(piece=-8192), dict(piece=100)):
        assert call(head(**bad)) == INVALID, bad
    assert call(None) == INVALID
    wide = dict(d=64, ldh=4096, ldw=4096)
    for bad in (dict(h=PTR + 1), dict(W=PTR + 1), dict(target=PTR + 4), dict(B=65536), dict(T=(1 << 30) + 1), dict(T=1 << 30, B=4),
                dict(V=(1 << 30) + 1), dict(dtype=dprc.F32, h=PTR + 2), dict(T=1 << 29, V=1 << 15), dict(T=1 << 29, d=1 << 12)):
        kw = dict(wide, **bad)
        if call is clip:
            assert call(head(**kw), ldg=1 << 31) == UNSUPPORTED, bad
        elif call is back:
            assert call(head(**kw), lddh=4096, lddw=4096) == UNSUPPORTED, bad
        else:
            assert call(head(**kw)) == UNSUPPORTED, bad
    assert call(head(d=1 << 21, ldh=1 << 21, ldw=1 << 21, V=1 << 20), **(
        dict(lddh=1 << 21, lddw=1 << 21) if call is back else dict(ldg=1 << 20) if call is clip else {})) == UNSUPPORTED


@built
def test_head_arguments():
    H = head()
    L = dprc.lib()
    assert loss(H, loss=0) == loss(H, lse=0) == loss(H, lse=4 * PTR) == loss(H, ws=0) == loss(H, ws=PTR + 8) == INVALID
    assert loss(H, loss=4 * PTR + 2) == UNSUPPORTED
    assert loss(H, n=L.dprc_head_loss_workspace(H) - 1) == SMALL
    assert errors(H, lse=0) == errors(H, g=0) == errors(H, E=0) == errors(H, v0=-1) == errors(H, nv=0) == INVALID
    assert errors(H, v0=291) == errors(H, nv=301, lde=301) == errors(H, lde=9) == INVALID
    assert errors(head(ldh=65), ws=0) == INVALID and errors(head(ldh=65), n=8) == SMALL
    assert errors(H, E=PTR) == errors(H, E=2 * PTR) == INVALID
    assert errors(H, E=6 * PTR + 1) == UNSUPPORTED
    assert back(H, lse=0) == back(H, g=0) == back(H, dh=0, dW=0) == back(H, lddh=63) == back(H, lddw=63) == INVALID
    assert back(H, dh=PTR) == back(H, dW=2 * PTR) == back(H, dW=6 * PTR) == back(H, ws=0) == INVALID
    assert back(H, dh=6 * PTR + 1) == back(H, g=5 * PTR + 2) == UNSUPPORTED
    for kw, want in ((dict(k=0), INVALID), (dict(k=257), INVALID), (dict(n2=0), INVALID), (dict(probe=3), INVALID),
                     (dict(side=3), INVALID), (dict(probe=2, k=33), UNSUPPORTED), (dict(n2=9 * PTR + 2), UNSUPPORTED)):
        assert back(H, nm=norms(**kw)) == want, kw
    for args in ((1, 1, None), (1, 0, None), (0, 1, None), (0, 0, norms()), (1, 1, norms())):
        need = L.dprc_head_backward_workspace(H, *args)
        assert need > 0
        assert back(H, dh=args[0] and 6 * PTR, dW=args[1] and 7 * PTR, nm=args[2], n=need - 1) == SMALL
    assert clip(H, lse=0) == clip(H, g=0) == clip(H, c=0) == clip(H, grad=0) == clip(H, ldg=299) == clip(H, ws=0) == INVALID
    assert clip(H, n=L.dprc_head_clip_accumulate_workspace(H) - 1) == SMALL
    assert L.dprc_head_loss_workspace(head(B=0)) == L.dprc_head_backward_workspace(head(d=0), 1, 1, None) == 0


@built
def test_head_workspace_is_bounded():
    """No more than about 1 GiB of E however large the vocabulary, and what `piece` says."""
    L = dprc.lib()
    H = lambda **kw: head(**dict(dict(B=8, T=4096, d=2048, ldh=2048, ldw=2048, V=128256), **kw))
    rows, planes = 8 * 4096 * (2048 * 2 + 4), 8 * 4096 * 2048 * 4
    assert L.dprc_head_backward_workspace(H(), 1, 0, None) <= (1 << 30) + rows + planes + 1024
    assert L.dprc_head_backward_workspace(H(piece=8192), 1, 0, None) <= (1 << 29) + rows + planes + 1024
    assert L.dprc_head_loss_workspace(H()) <= 8 * 4096 * 8 * 502


def rope(**kw):
    f = dict(B=2, T=8, D=64, r=32, freqs=PTR, pos=0, start=0, scale=1.0, interleaved=0, inverse=0, xdtype=1, ydtype=1)
    f.update(kw)
    return dprc.ROPE.pack(*f.values())


def heads(x=2 * PTR, y=3 * PTR, H=4, xb=2048, xt=256, xh=64, yb=2048, yt=256, yh=64):
    return [x, y, H, xb, xt, xh, yb, yt, yh]


def rotary(R, *hs, count=None):
    words = (ctypes.c_int64 * max(1, 9 * len(hs)))(*[w for h in hs for w in h])
    return dprc.lib().dprc_rotary(R, words, len(hs) if count is None else count, None)


@built
def test_rotary_refusals():
    ok = heads()
    for bad in (dict(B=0), dict(T=0), dict(D=0), dict(r=0), dict(r=33), dict(r=2 ** 31 - 1), dict(freqs=0), dict(xdtype=5), dict(ydtype=-1),
                dict(scale=math.inf), dict(scale=math.nan)):
        assert rotary(rope(**bad), ok) == INVALID, bad
    for bad in (dict(B=1 << 32), dict(B=1 << 16, T=1 << 16), dict(D=(1 << 20) + 2), dict(D=1 << 14, r=4097), dict(freqs=PTR + 4), dict(pos=PTR + 4)):
        assert rotary(rope(**bad), ok) == UNSUPPORTED, bad
    assert rotary(None, ok) == rotary(rope()) == rotary(rope(), ok, count=-1) == INVALID
    assert rotary(rope(), *[ok] * 5) == UNSUPPORTED
    for bad in (dict(x=0), dict(y=0), dict(H=0), dict(y=2 * PTR, yt=512), dict(y=2 * PTR, yh=65), dict(y=2 * PTR, yb=1)):
        assert rotary(rope(), heads(**bad)) == INVALID, bad
    assert rotary(rope(ydtype=0), heads(y=2 * PTR)) == INVALID
    for bad in (dict(x=PTR + 1), dict(y=PTR + 1), dict(H=(1 << 16) + 1)):
        assert rotary(rope(), heads(**bad)) == UNSUPPORTED, bad
    assert rotary(rope(), heads(H=1 << 16), heads(x=4 * PTR, y=5 * PTR, H=1)) == UNSUPPORTED
    assert rotary(rope(D=1 << 15, r=16), heads(H=1 << 15), heads(x=4 * PTR, y=5 * PTR, H=1)) == UNSUPPORTED
    # a result over another tensor, or over another result
    assert rotary(rope(), ok, heads(x=4 * PTR, y=2 * PTR)) == rotary(rope(), ok, heads(x=4 * PTR, y=3 * PTR)) == INVALID


def tensors(*ts):
    f = dict(x=PTR, out=2 * PTR, rows=3, cols=5, ldx=5, ldo=5, dtype=1)
    ts = [dict(f, **t) for t in ts]
    return b"".join(dprc.TENSOR.pack(*t.values()) for t in ts), len(ts)


@built
def test_joint_norm_refusals():
    L = dprc.lib()
    cl = lambda *ts, m=1.0, norm=PTR, ws=PTR, n=BIG: L.dprc_grad_clip(*tensors(*ts), m, norm, ws, n, None)
    no = lambda *ts, norm=PTR, ws=PTR, n=BIG: L.dprc_grad_norm(*tensors(*ts), norm, ws, n, None)
    for f in (cl, no):
        for bad in (dict(x=0), dict(rows=-1), dict(cols=-1), dict(ldx=4), dict(dtype=2)):
            assert f({}, bad) == INVALID, bad
        for bad in (dict(x=PTR + 1), dict(dtype=0, x=PTR + 2), dict(rows=1 << 41), dict(rows=1, cols=1 << 41)):
            assert f({}, bad) == UNSUPPORTED, bad
        assert f({}, ws=0) == f({}, ws=PTR + 8) == INVALID
        assert f({}, n=L.dprc_grad_norm_workspace(*tensors({})) - 1) == SMALL
        assert f({}, norm=PTR + 2) == UNSUPPORTED
    for bad in (dict(out=0), dict(ldo=4), dict(out=PTR, ldo=6)):
        assert cl({}, bad) == INVALID, bad
    for m in (0.0, -1.0, math.inf, math.nan):
        assert cl({}, m=m) == INVALID
    assert no({}, norm=0) == INVALID
    assert L.dprc_grad_norm(None, 1, PTR, PTR, BIG, None) == L.dprc_grad_norm(None, -1, PTR, PTR, BIG, None) == INVALID


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def entry(name):
        if name.endswith("_workspace"):
            return lambda *a: 0
        return lambda *a: seen.append((name, a)) or dprc.SUCCESS
    monkeypatch.setattr(dprc, "lib", lambda: types.SimpleNamespace(**{n: entry(n) for n in dprc.EXPORTS}))
    monkeypatch.setattr(dprc, "_stream", lambda dev: None)
    return seen


def test_binding_refuses_mismatched_head_tensors(calls):
    h, W, y, s = torch.zeros(2, 3, 8), torch.zeros(11, 8), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3)
    ok = dict(h=h, W=W, target=y)
    for bad in (dict(h=h[0]), dict(h=h.double()), dict(h=torch.zeros(2, 3, 16)[..., ::2]), dict(W=W[:, :7]), dict(W=W.bfloat16()),
                dict(W=torch.zeros(8, 11).t()), dict(W=W[0]), dict(target=y.int()), dict(target=y[:1]), dict(target=y.view(-1)),
                dict(target=torch.zeros(2, 6, dtype=torch.int64)[:, ::2])):
        with pytest.raises((ValueError, TypeError)):
            dprc.dprc_head_loss(**dict(ok, **bad))
    for bad in (dict(loss=torch.zeros(6)), dict(lse=s.double()), dict(loss=torch.zeros(2, 6)[:, ::2]), dict(lse=torch.zeros(2, 4))):
        with pytest.raises(ValueError):
            dprc.dprc_head_loss(**ok, **bad)
    for bad in (dict(lse=s[:1]), dict(g=s.t()), dict(g=torch.zeros(1).expand(2, 3)), dict(dh=torch.zeros(2, 3, 7)), dict(dh=h.bfloat16()),
                dict(dW=torch.zeros(11, 7)), dict(dW=torch.zeros(8, 11).t()), dict(n2=torch.zeros(3), k=4), dict(n2=torch.zeros(1).expand(2), k=4)):
        with pytest.raises(ValueError):
            dprc.dprc_head_backward(**dict(dict(ok, lse=s, g=s), **bad))
    for bad in (dict(c=torch.zeros(3)), dict(c=torch.zeros(1).expand(2)), dict(grad=torch.zeros(8, 10)), dict(grad=torch.zeros(8, 11).double()),
                dict(grad=torch.zeros(11, 8).t())):
        with pytest.raises(ValueError):
            dprc.dprc_head_clip_accumulate(**dict(dict(ok, lse=s, g=s, c=torch.zeros(2)), **bad))
    for bad in (dict(E=torch.zeros(2, 3, 10)), dict(E=torch.zeros(2, 3, 11).bfloat16())):
        with pytest.raises(ValueError):
            dprc.dprc_head_errors(**ok, lse=s, g=s, **bad)
    assert not calls


def test_binding_refuses_mismatched_heads(calls):
    x, f = torch.zeros(2, 3, 4, 8), torch.zeros(4, dtype=torch.float64)
    for bad in (dict(x=x[0]), dict(x=[]), dict(x=x.double()), dict(x=[x, x.bfloat16()]), dict(x=[x, x[:1]]), dict(x=[x, x[..., :6]]),
                dict(x=torch.zeros(2, 3, 4, 16)[..., ::2]), dict(freqs=f.float()), dict(freqs=f[:, None]), dict(freqs=torch.zeros(8).double()[::2]),
                dict(pos=torch.zeros(2, 3)), dict(pos=torch.zeros(3, dtype=torch.int64)), dict(pos=torch.zeros(1, 3, dtype=torch.int64).expand(2, 3)),
                dict(out=torch.zeros(2, 3, 4, 1).expand(2, 3, 4, 8)), dict(out=torch.zeros(1, 3, 4, 8).expand(2, 3, 4, 8)), dict(out=x[:1]),
                dict(out=[x, x]), dict(x=[x, x], out=[x, x]), dict(out_dtype=torch.float16)):
        with pytest.raises((ValueError, TypeError)):
            dprc.dprc_rotary(**dict(dict(x=x, freqs=f), **bad))
    assert not calls
    y = dprc.dprc_rotary(x, f, heads_first=True)
    assert y.shape == x.shape and y.stride() == (96, 8, 24, 1)


def test_binding_refuses_mismatched_tensors(calls):
    a, b = torch.zeros(4, 5), torch.zeros(7)
    for ts, kw in (([], {}), ([a.t()], {}), ([a.double()], {}), ([a, b], dict(outs=[a])), ([a, b], dict(outs=[a, a])), ([a, a], {}),
                   ([a], dict(outs=[a.bfloat16()])), ([a], dict(outs=[b])), ([a], dict(outs=[torch.zeros(5, 4).t()])),
                   ([b[::2]], {}), ([torch.zeros(1, 5).expand(4, 5)], {}), ([a], dict(norm=torch.zeros(2)))):
        with pytest.raises((ValueError, TypeError)):
            dprc.dprc_grad_clip(ts, 1.0, **kw)
    assert not calls
    wide = torch.zeros(4, 9)[:, :5]
    with pytest.raises(ValueError, match="another"):
        dprc.dprc_grad_clip([a, wide], 1.0, outs=[wide, a])
    assert not calls
    dprc.dprc_grad_clip([a, wide], 1.0, outs=[torch.zeros(4, 9)[:, :5], torch.zeros(4, 5)])
    assert calls[-1][0] == "dprc_grad_clip" and calls[-1][1][1] == 2
    words = dprc._tensors([a, wide, a], [torch.zeros(4, 9)[:, :5], torch.zeros(4, 5), torch.zeros(4, 5)])   # rows, columns, row strides
    assert [t[2:6] for t in dprc.TENSOR.iter_unpack(words)] == [(4, 5, 5, 9), (4, 5, 9, 5), (1, 20, 20, 20)]


@pytest.mark.parametrize("R,C,wide", [(2, 4, 8), (2, 1, 2), (3, 5, 15), (3, 5, 7), (3, 5, 5 * 15)])
def test_rows_beside_a_contiguous_tensor_keep_their_stride(calls, R, C, wide):
    """A matrix whose rows lie any number of elements apart (its own number of elements, too) beside a contiguous one, as
    the tensor or as the result, is packed with both strides."""
    t, rows = torch.ones(R, C), torch.zeros(R, wide)[:, :C]
    shape = lambda *a: [w[2:6] for w in dprc.TENSOR.iter_unpack(dprc._tensors(*a))]
    assert shape([t], [rows]) == [(R, C, C, wide)]
    assert shape([rows], [t]) == [(R, C, wide, C)]
    assert shape([rows], [torch.zeros(R, wide + 1)[:, :C]]) == [(R, C, wide, wide + 1)]
    assert shape([rows], None) == [(R, C, wide, wide)]
    assert shape([t], [torch.zeros(R, C)]) == [(1, R * C, R * C, R * C)]


def test_binding_refuses_a_result_over_another_entrys_tensor(calls):
    """A tensor listed twice may be scaled in place by neither entry: the other one still reads it."""
    a, b, e = torch.ones(4, 5), torch.ones(4, 5), torch.zeros(0)
    rows = torch.ones(4, 9)[:, :5]
    for ts, outs in (([a, a], [a, b]), ([a, a], [b, a]), ([a, rows, rows], [b, rows, torch.ones(4, 5)]), ([e, e, a, a], [e, e, a.view(4, 5), b])):
        with pytest.raises(ValueError, match="another"):
            dprc.dprc_grad_clip(ts, 1.0, outs=outs)
    assert not calls
    dprc.dprc_grad_clip([a, a], 1.0, outs=[b, torch.ones(4, 5)])        # read twice, written elsewhere
    dprc.dprc_grad_clip([e, a, e, b], 1.0, outs=[e, a, torch.zeros(0), torch.ones(4, 5)])
    assert len(calls) == 2


def test_oracle_against_torch():
    rng = np.random.default_rng(0)
    h, W = rng.standard_normal((2, 5, 7)), rng.standard_normal((11, 7))
    y = rng.integers(0, 11, (2, 5))
    y[0, 1] = -100
    ht, Wt = torch.tensor(h, requires_grad=True), torch.tensor(W, requires_grad=True)
    ref = torch.nn.functional.cross_entropy((ht @ Wt.t()).view(-1, 11), torch.tensor(y).view(-1), reduction="none").view(2, 5)
    l, z = O.loss(h, W, y)
    np.testing.assert_allclose(l, ref.detach().numpy(), rtol=1e-12)
    g = rng.standard_normal((2, 5))
    (ref * torch.tensor(g)).sum().backward()
    E = O.errors(h, W, y, z, g)
    np.testing.assert_allclose(E @ W, ht.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(E.reshape(-1, 11).T @ h.reshape(-1, 7), Wt.grad.numpy(), atol=1e-12)
    x = rng.standard_normal((2, 5, 3, 8))
    f, pos = np.array([1.0, 0.1, 0.01]), rng.integers(0, 100, (2, 5))
    for inter in (False, True):
        y1 = O.rotary(x, f, pos, 1.5, inter)
        np.testing.assert_allclose(O.rotary(y1, f, pos, 1 / 1.5, inter, True), x, atol=1e-12)
        z1 = torch.view_as_complex(torch.tensor(x[..., :6].reshape(2, 5, 3, 3, 2) if inter else np.stack([x[..., :3], x[..., 3:6]], -1)))
        w = z1 * torch.polar(torch.full((2, 5, 1, 3), 1.5, dtype=torch.float64), torch.tensor(pos[:, :, None, None] * f))
        got = torch.view_as_real(w).numpy()
        np.testing.assert_allclose(y1[..., :6], got.reshape(2, 5, 3, 6) if inter else np.concatenate([got[..., 0], got[..., 1]], -1), atol=1e-12)
    (c,), n = O.clip([np.array([3.0, 4.0])], 1.0)
    assert n == 5.0 and np.allclose(c, [0.6, 0.8])
