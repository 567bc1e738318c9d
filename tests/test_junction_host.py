"""Host-side checks of the dropout, norm and vector entry points (no GPU): arguments are refused
before anything is enqueued, by the library and by the binding."""

import ctypes
import os
import types

import pytest
import torch

from paper_2605_24879_amd import dprc
from paper_2605_24879_amd.junction import token_rows

pytestmark = pytest.mark.skipif(not os.path.exists(dprc.LIB_PATH), reason="libdprc.so not built")

X, Z, S, Y, M, RS, W, WS = (0x10000 * (j + 1) for j in range(8))
BAD, UNSUPPORTED, SMALL = 1, 2, 3


def ln(**kw):
    a = dict(dict(B=2, T=32, n=64, dtype=dprc.BF16, wdtype=dprc.BF16, kind=0, eps=1e-5, weight=W, bias=W, p=0.1,
                  site_id=0, seed=0), **kw)
    return dprc.LN(*(a[k] for k, _ in dprc.LN._fields_))


def test_struct_layout():
    assert ctypes.sizeof(dprc.LN) == 72 and dprc.LN.weight.offset == 40 and dprc.LN.seed.offset == 64


def test_dropout_validation():
    def call(x=X, ldx=64, res=Z, ldr=64, out=S, ldo=64, rows=8, n=64, dt=dprc.BF16, p=0.1):
        return dprc.lib().dprc_dropout(x, ldx, res, ldr, out, ldo, rows, n, dt, p, 0, 0, None)
    for kw in (dict(x=0), dict(out=0), dict(rows=0), dict(n=0), dict(rows=-1), dict(dt=7), dict(ldx=63), dict(ldr=63),
               dict(ldo=63), dict(p=-0.1), dict(p=1.1), dict(p=float("nan"))):
        assert call(**kw) == BAD, kw
    for kw in (dict(x=X + 1), dict(res=Z + 1), dict(out=S + 1), dict(dt=dprc.F32, x=X + 2), dict(rows=(1 << 31) + 1),
               dict(n=1 << 31, ldx=1 << 31, ldr=1 << 31, ldo=1 << 31)):
        assert call(**kw) == UNSUPPORTED, kw


def test_layernorm_validation():
    def call(L=None, x=X, ldx=64, res=Z, ldr=64, s=S, lds=64, y=Y, ldy=64, mean=M, rstd=RS, **kw):
        L = ctypes.byref(ln(**kw)) if L is None else L
        return dprc.lib().dprc_layernorm(L, x, ldx, res, ldr, s, lds, y, ldy, mean, rstd, None)
    assert dprc.lib().dprc_layernorm(None, X, 64, None, 0, None, 0, Y, 64, None, None, None) == BAD
    for kw in (dict(B=0), dict(T=0), dict(n=0), dict(n=-5), dict(dtype=4), dict(wdtype=-1), dict(kind=2), dict(eps=0.0),
               dict(eps=float("inf")), dict(eps=float("nan")), dict(p=-1.0), dict(p=2.0), dict(x=0), dict(y=0),
               dict(ldx=63), dict(ldr=63), dict(lds=63), dict(ldy=63), dict(s=Y)):
        assert call(**kw) == BAD, kw
    big = 1 << 31
    for kw in (dict(x=X + 1), dict(res=Z + 1), dict(s=S + 1), dict(y=Y + 1), dict(weight=W + 1), dict(bias=W + 1),
               dict(mean=M + 2), dict(rstd=RS + 2), dict(dtype=dprc.F32, y=Y + 2), dict(wdtype=dprc.F32, weight=W + 2),
               dict(B=1 << 20, T=1 << 20), dict(n=big, ldx=big, ldr=big, lds=big, ldy=big)):
        assert call(**kw) == UNSUPPORTED, kw


def test_layernorm_backward_validation():
    lib = dprc.lib()

    def call(dy=X, ldd=64, s=S, lds=64, mean=M, rstd=RS, ds=Z, ldds=64, dx=Y, lddx=64, dh=Y + 0x8000, lddh=64, dw=0x90000,
             db=0xA0000, ldg=64, ws=WS, ws_bytes=1 << 30, **kw):
        return lib.dprc_layernorm_backward(ctypes.byref(ln(**kw)), dy, ldd, s, lds, mean, rstd, ds, ldds, dx, lddx, dh, lddh,
                                           dw, db, ldg, ws, ws_bytes, None)
    for kw in (dict(B=0), dict(n=0), dict(dtype=4), dict(kind=5), dict(p=1.5), dict(dy=0), dict(s=0), dict(rstd=0), dict(mean=0),
               dict(dx=0, dh=0, dw=0, db=0), dict(ldd=63), dict(lds=63), dict(ldds=63), dict(lddx=63), dict(lddh=63),
               dict(ldg=63), dict(dh=Y), dict(db=0x90000)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dy=X + 1), dict(s=S + 1), dict(ds=Z + 1), dict(dx=Y + 1), dict(dh=Y + 1), dict(weight=W + 1),
               dict(mean=M + 1), dict(rstd=RS + 2), dict(dw=0x90002), dict(db=0xA0001), dict(T=1 << 31)):
        assert call(**kw) == UNSUPPORTED, kw
    # a long sample's tokens are split, which needs the workspace (with weight or bias gradients only)
    L = ln(B=1, T=32768, n=2048, weight=None, bias=None)
    need = lib.dprc_layernorm_backward_workspace(ctypes.byref(L))
    assert need > 0
    long = dict(B=1, T=32768, n=2048, ldd=2048, lds=2048, ldds=2048, lddx=2048, lddh=2048, ldg=2048)
    assert call(ws_bytes=need - 1, **long) == SMALL
    assert call(ws=0, ws_bytes=need, **long) == BAD
    assert call(ws=WS + 16, ws_bytes=need, **long) == BAD
    for kw in (dict(B=0), dict(kind=3), dict(n=0), dict(p=-1.0), dict(T=1 << 31)):
        assert lib.dprc_layernorm_backward_workspace(ctypes.byref(ln(**kw))) == 0, kw
    assert lib.dprc_layernorm_backward_workspace(None) == 0


def test_vector_validation():
    lib = dprc.lib()
    norm = lambda G=X, ldg=64, B=2, n=64, out=Y, ws=WS, wb=1 << 30: lib.dprc_norm_vectors(G, ldg, B, n, out, 0, ws, wb, None)
    acc = lambda G=X, ldg=64, c=Z, B=2, n=64, out=Y, ws=WS, wb=1 << 30: lib.dprc_clip_accumulate_vectors(
        G, ldg, c, B, n, out, 0, ws, wb, None)
    for f in (norm, acc):
        for kw in (dict(G=0), dict(out=0), dict(B=0), dict(n=0), dict(ldg=63)):
            assert f(**kw) == BAD, kw
        for kw in (dict(G=X + 2), dict(out=Y + 1), dict(B=(1 << 24) + 1), dict(n=1 << 41, ldg=1 << 41)):
            assert f(**kw) == UNSUPPORTED, kw
    assert acc(c=0) == BAD and acc(c=Z + 1) == UNSUPPORTED
    for q, f, B, n in ((lib.dprc_norm_vectors_workspace, norm, 2, 1 << 22),
                       (lib.dprc_clip_accumulate_vectors_workspace, acc, 1 << 16, 64)):
        assert q(0, 64) == 0 and q(2, 0) == 0
        need = q(B, n)
        if need:
            assert f(B=B, n=n, ldg=n, wb=need - 1) == SMALL
            assert f(B=B, n=n, ldg=n, ws=0, wb=need) == BAD
            assert f(B=B, n=n, ldg=n, ws=WS + 8, wb=need) == BAD


@pytest.fixture
def no_launch(monkeypatch):
    """A library of which no entry point but the workspace queries may be reached."""
    monkeypatch.setattr(dprc, "lib", lambda: types.SimpleNamespace(
        **{n: (lambda *a, n=n: 0 if n.endswith("_workspace") else pytest.fail(n)) for n in dprc.EXPORTS}))


def test_the_binding_refuses_what_the_kernels_cannot_take(no_launch):
    x, v, st = torch.zeros(2, 3, 8), torch.zeros(8), torch.zeros(6)
    G = torch.zeros(2, 8)
    meta = torch.zeros(2, 3, 8, device="meta")
    calls = [
        # host tensors have no stream
        lambda: dprc.dprc_dropout(x, 0.1, 0, 0), lambda: dprc.dprc_layernorm(x, v),
        lambda: dprc.dprc_layernorm_backward(x, x, v, st, st),
        lambda: dprc.dprc_norm_vectors(G), lambda: dprc.dprc_clip_accumulate_vectors(G, torch.zeros(2)),
        # shapes, strides, types, devices
        lambda: dprc.dprc_dropout(x[0], 0.1, 0, 0), lambda: dprc.dprc_dropout(x.transpose(1, 2), 0.1, 0, 0),
        lambda: dprc.dprc_dropout(x[:, ::2], 0.1, 0, 0), lambda: dprc.dprc_dropout(x, 0.1, 0, 0, res=x[:, :2]),
        lambda: dprc.dprc_dropout(x, 0.1, 0, 0, res=x.double()), lambda: dprc.dprc_dropout(x, 0.1, 0, 0, res=meta),
        lambda: dprc.dprc_dropout(x, 0.1, 0, 0, out=x[:, :, :4]), lambda: dprc.dprc_dropout(x.double(), 0.1, 0, 0),
        lambda: dprc.dprc_layernorm(x, v[:7]), lambda: dprc.dprc_layernorm(x, v, v.double()),
        lambda: dprc.dprc_layernorm(x, torch.zeros(16)[::2]), lambda: dprc.dprc_layernorm(x, meta[0, 0]),
        lambda: dprc.dprc_layernorm(x, v, res=x[:1]), lambda: dprc.dprc_layernorm(x, v, y=x.bfloat16()),
        lambda: dprc.dprc_layernorm_backward(x, x[:, :2], v, st, st),
        lambda: dprc.dprc_layernorm_backward(x, x, v, st[:5], st), lambda: dprc.dprc_layernorm_backward(x, x, v, st, st.double()),
        lambda: dprc.dprc_layernorm_backward(x, x, v, st, st, ds=x.bfloat16()),
        lambda: dprc.dprc_layernorm_backward(x, x, v, st, st, dw=G.double()),
        lambda: dprc.dprc_layernorm_backward(x, x, v, st, st, dw=G, db=torch.zeros(2, 16)[:, :8]),
        lambda: dprc.dprc_norm_vectors(G.t()), lambda: dprc.dprc_norm_vectors(G.double()),
        lambda: dprc.dprc_norm_vectors(G, n2=torch.zeros(3)), lambda: dprc.dprc_clip_accumulate_vectors(G, torch.zeros(3)),
        lambda: dprc.dprc_clip_accumulate_vectors(G, torch.zeros(2), grad=torch.zeros(9)),
    ]
    for k, call in enumerate(calls):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"call {k} was taken")


def test_token_rows_copies_only_what_has_no_row_stride():
    x = torch.randn(4, 6, 10)
    keeps = {"whole": x, "last tokens": x[:, -1:], "one sample's part": x[1:2, 2:5], "one row": x[3:, 5:], "columns": x[:, :, 2:7],
             "last tokens' columns": x[:, -1:, 3:], "every other sample's token": x[::2, :1]}
    copies = {"cut tokens": x[:, 1:4], "features apart": x[:, :, ::2], "tokens first": x.transpose(0, 1), "spread": x[:1, :1].expand(4, 6, 10),
              "spread samples": x[:1, :1].expand(4, 1, 10)}
    for name, v in keeps.items():
        assert token_rows(v) is v, name
    for name, v in copies.items():
        got = token_rows(v)
        assert got is not v and got.is_contiguous() and torch.equal(got, v), name
    for v in (*keeps.values(), *map(token_rows, copies.values())):
        assert dprc._token_rows(v, "x") >= v.shape[2]
