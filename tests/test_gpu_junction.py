"""Dropout, residual sum, norm, their gradients and the norms' private gradients against the
64-bit oracle.

Tolerances, with u = 2^-24 (rounding to fp32) and r = 2^-8 (to bf16: 8 significant bits; 0 for fp32 outputs):

* dropout: one product and one sum, u (2 |x f| + 2 |out|), and the output's r |out|;
* sums over a row of n terms: no partial sum is a chain of more than K = max(64, n / 64) roundings,
  so a sum is off by at most K u times the sum of its terms' magnitudes;
* y: the mean is off by m = K u mean|s| (and s itself by 2 u (|x f| + |res|)), the variance,
  taken about that mean, by K u of itself and m^2, so rstd by e = (K + 8) u + (m rstd)^2 of itself;
  y by |w| (m rstd + |xh| e) + 4 u (|w xh| + |b|) + r |y|;
* dx: xh by 2 u |xh| + u rstd (|s| + |mu|) through the subtraction, the row means by (K + 4) u of
  their terms' mean magnitudes: rstd ((8 u) (|g| + ...) + ...) + 2 u |dx| + r |dx|;
* dw, db: sums over T tokens, at most T + 8 roundings in a chain, and the terms' own errors;
* squared norms: the terms and their sum are exact to 64 bits, u of the sum (2 u accumulated);
* clipped sums: chains of at most B + 2 roundings.

A dropped element has to be exactly zero (the residual exactly, where there is one).
"""

import numpy as np
import pytest
import torch

from oracle import junction as J
from oracle.estimators import as_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SEED, SITE, EPS = 0xFEDCBA9876543210, 3, 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
R = {"bf16": 2.0 ** -8, "f32": 0.0}


@pytest.fixture(scope="module")
def D():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc
    dprc.lib()
    return dprc


def rows(B, T, n, dtype, seed, pad=0, scale=1.0, shift=0.0):
    """[B, T, n] token rows of stride n + pad; what lies between the rows is NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((B, T, n + pad), float("nan"))
    x[..., :n] = scale * torch.randn(B, T, n, generator=g) + shift
    return x.to(DT[dtype]).cuda()[..., :n]


def vec(n, dtype, seed, scale=0.1, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (shift + scale * torch.randn(n, generator=g)).to(DT[dtype]).cuda()


def within(got, ref, tol):
    got = as_f64(got)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - ref) - tol)), np.argwhere(bad)[:4].tolist())


# ---- dropout -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("B,T,n,pad", [(1, 1, 1, 0), (1, 3, 2, 1), (3, 5, 7, 0), (2, 64, 64, 0), (2, 33, 111, 2),
                                       (1, 300, 200, 0), (1, 2, 2049, 0), (4, 61, 1111, 3), (2, 3, 8200, 8)])
def test_dropout(D, B, T, n, pad, res, dtype):
    x, z = rows(B, T, n, dtype, 1, pad), rows(B, T, n, dtype, 2, pad) if res else None
    for p in (0.0, 0.1, 0.5, 1.0):
        got = D.dprc_dropout(x, p, SEED, SITE, res=z)
        ref = J.dropout(x, SEED, SITE, p, res=z)
        xf = np.abs(J.dropout(x, SEED, SITE, p))
        within(got, ref, U * (2 * xf + 2 * np.abs(ref)) + R[dtype] * np.abs(ref))
        dropped = torch.from_numpy(J.dropout_factors(SEED, SITE, B * T, n, p).reshape(B, T, n) == 0).cuda()
        assert torch.equal(got[dropped], z[dropped] if res else torch.zeros_like(got[dropped]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_elements_are_zero_whatever_they_were(D, dtype):
    x = rows(2, 16, 120, dtype, 3)
    dropped = torch.from_numpy(J.dropout_factors(SEED, SITE, 32, 120, 0.3).reshape(2, 16, 120) == 0).cuda()
    bad = x.clone()
    bad[dropped] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda", dtype=x.dtype).repeat(
        (int(dropped.sum()) + 2) // 3)[:int(dropped.sum())]
    assert torch.equal(D.dprc_dropout(bad, 0.3, SEED, SITE), D.dprc_dropout(x, 0.3, SEED, SITE))
    assert torch.equal(D.dprc_dropout(bad, 1.0, SEED, SITE, res=x), x)
    y0, s0, _, _ = D.dprc_layernorm(x, p=0.3, seed=SEED, site_id=SITE)
    y1, s1, _, _ = D.dprc_layernorm(bad, p=0.3, seed=SEED, site_id=SITE)
    assert torch.equal(y0, y1) and torch.equal(s0, s1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropout_in_place_and_on_views(D, dtype):
    x, z = rows(2, 9, 75, dtype, 4), rows(2, 9, 75, dtype, 5)
    ref = D.dprc_dropout(x, 0.2, SEED, SITE, res=z)
    a, b = x.clone(), z.clone()
    assert torch.equal(D.dprc_dropout(a, 0.2, SEED, SITE, res=z, out=a), ref)
    assert torch.equal(D.dprc_dropout(x, 0.2, SEED, SITE, res=b, out=b), ref)
    wide = torch.full((2, 9, 200), 7.0, dtype=DT[dtype], device="cuda")
    for c0 in (0, 1, 3, 8, 125):                                     # bases at every alignment of an element
        out = wide.clone()
        out[:, :, c0:c0 + 75] = x
        D.dprc_dropout(out[:, :, c0:c0 + 75], 0.2, SEED, SITE, res=z, out=out[:, :, c0:c0 + 75])
        assert torch.equal(out[:, :, c0:c0 + 75], ref)
        assert (out[:, :, :c0] == 7.0).all() and (out[:, :, c0 + 75:] == 7.0).all()


# ---- forward --------------------------------------------------------------------------------------

def check_forward(D, x, z, w, b, p, kind, eps=EPS, **kw):
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    rms = kind == D.RMSNORM
    n = x.shape[-1]
    y, s, mean, rstd = D.dprc_layernorm(x, w, b, eps=eps, kind=kind, res=z, p=p, seed=SEED, site_id=SITE, **kw)
    s64 = J.dropout(x, SEED, SITE, p, res=z)
    ry, rm, rr = J.norm(s64, w, b, eps=eps, rms=rms)
    K = max(64, n / 64)
    xf = np.abs(J.dropout(x, SEED, SITE, p))
    ds = U * (2 * xf + 2 * np.abs(s64))
    if z is not None or p > 0:
        within(s, s64, ds + R[dtype] * np.abs(s64))
    else:
        assert s.data_ptr() == x.data_ptr()
    m = np.zeros(s64.shape[:-1] + (1,)) if rms else K * U * np.abs(s64).mean(-1, keepdims=True) + ds.mean(-1, keepdims=True)
    r3 = rr.reshape(s64.shape[:-1] + (1,))
    e = (K + 8) * U + (m * r3) ** 2 + (2 * ds * r3).max(-1, keepdims=True)
    w64 = np.ones(n) if w is None else as_f64(w)
    b64 = np.zeros(n) if b is None else as_f64(b)
    xh = (s64 - (0 if rms else rm.reshape(r3.shape))) * r3
    tol = np.abs(w64) * ((m + ds + U * np.abs(s64)) * r3 + np.abs(xh) * e) + 4 * U * (np.abs(w64 * xh) + np.abs(b64))
    within(y, ry, tol + R[dtype] * np.abs(ry))
    within(rstd, rr, (rr.reshape(r3.shape) * e).reshape(-1) + U * rr)
    if rms:
        assert mean is None
    else:
        within(mean, rm, m.reshape(-1) + U * np.abs(rm))
    return y, s, mean, rstd


@pytest.mark.parametrize("kind", ["LAYERNORM", "RMSNORM"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 31, 63, 64, 65, 111, 128, 200, 256, 257, 500, 512, 513, 1000, 1024, 1025,
                               1111, 1536, 1537, 2048, 2049, 4000, 4096, 4097, 8192, 8200, 16384, 16391, 32768, 32776,
                               40003])
def test_norm_widths(D, n, dtype, kind):
    B, T = (2, 19) if n <= 4096 else (1, 3)
    x, z = rows(B, T, n, dtype, n, scale=0.5), rows(B, T, n, dtype, n + 1, shift=0.3)
    w, b = vec(n, dtype, n + 2, shift=1.0), vec(n, dtype, n + 3)
    check_forward(D, x, z, w, b, 0.1, getattr(D, kind))
    check_forward(D, x, None, w, None, 0.0, getattr(D, kind))


@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("B,T,n,pad", [(2, 13, 8193, 0), (1, 1, 8200, 1), (3, 20, 9001, 3), (5, 12, 12288, 0), (1, 40, 16383, 5),
                                       (1030, 1, 8196, 0)])
def test_backward_rows_of_a_whole_workgroup(D, B, T, n, pad, dtype, wdtype):
    # a row takes all threads of a workgroup; samples whole and cut, more of them than workgroups
    dy, s, ds = rows(B, T, n, dtype, 1, pad), rows(B, T, n, dtype, 2, pad, shift=0.5), rows(B, T, n, dtype, 3, pad)
    w = vec(n, wdtype, 4, shift=1.0)
    for k in (D.LAYERNORM, D.RMSNORM):
        check_backward(D, dy, s, w, k, ds, 0.25)
    check_backward(D, dy, s, None, D.LAYERNORM, None, 0.5, bias_grad=False)
    check_backward(D, dy, s, w, D.LAYERNORM, ds, 0.0, weight_grad=False)
    check_backward(D, dy, s, w, D.RMSNORM, None, 0.0, weight_grad=False, bias_grad=False)


@pytest.mark.parametrize("kind", ["LAYERNORM", "RMSNORM"])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("B,T,n,pad", [(1, 1, 64, 0), (1, 1, 2048, 0), (64, 1, 2048, 3), (1, 700, 64, 0), (5, 333, 111, 1),
                                       (2, 100, 2048, 8), (300, 3, 1111, 5)])
def test_norm_forms(D, B, T, n, pad, dtype, wdtype, kind):
    k = getattr(D, kind)
    x, z = rows(B, T, n, dtype, 1, pad, scale=0.5), rows(B, T, n, dtype, 2, pad)
    w, b = vec(n, wdtype, 3, shift=1.0), vec(n, wdtype, 4)
    for res in (None, z):
        for p in (0.0, 0.25):
            check_forward(D, x, res, w, b, p, k)
    check_forward(D, x, z, None, None, 0.0, k)
    check_forward(D, x, z, None, b, 0.0, k)
    check_forward(D, x, z, w, None, 1.0, k)


@pytest.mark.parametrize("n,rows_", [(64, 6000), (200, 3000), (2048, 1500), (5000, 700)])
def test_norm_of_many_rows(D, n, rows_):
    x, z = rows(1, rows_, n, "bf16", 1), rows(1, rows_, n, "bf16", 2)
    check_forward(D, x, z, vec(n, "bf16", 3, shift=1.0), None, 0.1, D.LAYERNORM)


def test_norm_is_fp32_before_its_one_rounding(D):
    # the norm is of the unrounded sum: beside a bf16 residual of 256 nearly all of the branch is rounded away,
    # the norm still sees it
    x = rows(1, 4, 512, "bf16", 1, scale=0.2)
    z = torch.full((1, 4, 512), 256.0, dtype=torch.bfloat16, device="cuda")
    y, s, _, _ = D.dprc_layernorm(x, res=z)
    ref, _, _ = J.norm(as_f64(x) + 256.0)
    assert torch.equal(s, (x.float() + z.float()).bfloat16())
    # sums of 256 +- 0.2 in fp32 are off by 2^-17 each (and so the mean at most), 2^-16 / 0.2 in xh
    within(y, ref, 2.0 ** -16 / 0.2 * 1.5 * (1 + np.abs(ref)) + R["bf16"] * np.abs(ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [8, 100, 2048, 5000])
def test_rows_without_spread(D, n, dtype):
    # zeros (padding), a constant (its variance is rounding only), one large entry
    x = torch.zeros(1, 4, n, dtype=DT[dtype], device="cuda")
    x[0, 1] = 3.0
    x[0, 2, n // 2] = 1000.0
    for kind in (D.LAYERNORM, D.RMSNORM):
        w, b = vec(n, dtype, 1, shift=1.0), vec(n, dtype, 2)
        y, _, mean, rstd = D.dprc_layernorm(x, w, b, eps=EPS, kind=kind)
        assert torch.equal(y[0, 0], b) and torch.equal(y[0, 3], b)
        assert torch.isfinite(y).all() and torch.isfinite(rstd).all()
        # 3 n is exact in fp32 and so is 3 n / n up to one rounding of 1 / n and one of the product
        ref, _, _ = J.norm(x, w, b, eps=EPS, rms=kind == D.RMSNORM)
        off = 3 * 2 * U / np.sqrt(EPS) * 1.2 if kind == D.LAYERNORM else 0.0
        within(y[0, 1], ref[0, 1], off * np.abs(as_f64(w)) + 100 * U * (1 + np.abs(ref[0, 1])) + R[dtype] * np.abs(ref[0, 1]))


def test_a_bad_row_stays_alone(D):
    for n in (64, 111, 2048, 5000):
        x, dy = rows(2, 9, n, "f32", 1), rows(2, 9, n, "f32", 2)
        bad = x.clone()
        bad[0, 3, n // 3] = float("nan")
        bad[1, 7, 0] = float("inf")
        y0, _, m0, r0 = D.dprc_layernorm(x)
        y1, _, m1, r1 = D.dprc_layernorm(bad)
        keep = torch.ones(2, 9, dtype=torch.bool, device="cuda")
        keep[0, 3] = keep[1, 7] = False
        assert torch.equal(y0[keep], y1[keep]) and torch.equal(r0.view(2, 9)[keep], r1.view(2, 9)[keep])
        assert torch.isnan(y1[0, 3]).all() and torch.isnan(y1[1, 7]).all()
        dx0 = D.dprc_layernorm_backward(dy, x, None, m0, r0)[0]
        dx1, _, dw1, db1 = D.dprc_layernorm_backward(dy, bad, None, m1, r1)
        assert torch.equal(dx0[keep], dx1[keep]) and torch.isnan(dx1[0, 3]).all()
        assert torch.isnan(dw1).all() and torch.isfinite(db1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [64, 75, 2048, 4097])
def test_norm_in_place_and_on_views(D, n, dtype):
    x, z, w = rows(2, 9, n, dtype, 1), rows(2, 9, n, dtype, 2), vec(n, dtype, 3, shift=1.0)
    call = lambda x, z, **kw: D.dprc_layernorm(x, w, res=z, p=0.1, seed=SEED, site_id=SITE, **kw)
    y, s, mean, rstd = call(x, z)
    a, b = x.clone(), z.clone()
    y1, s1, _, _ = call(a, b, y=a, s=b)
    assert y1 is a and s1 is b and torch.equal(a, y) and torch.equal(b, s)
    a, b = x.clone(), z.clone()
    call(a, b, y=b, s=a)
    assert torch.equal(b, y) and torch.equal(a, s)
    wide = torch.full((2, 9, 3 * n + 40), 7.0, dtype=DT[dtype], device="cuda")
    for c0 in (0, 1, 5, 8):
        out = wide.clone()
        yv, sv = out[:, :, c0:c0 + n], out[:, :, c0 + n + 11:c0 + 2 * n + 11]
        call(x, z, y=yv, s=sv)
        assert torch.equal(yv, y) and torch.equal(sv, s)
        yv.fill_(7.0), sv.fill_(7.0)
        assert (out == 7.0).all()


def test_norm_without_statistics_and_on_another_stream(D):
    x, w = rows(4, 33, 512, "bf16", 1), vec(512, "bf16", 2, shift=1.0)
    y, _, _, _ = D.dprc_layernorm(x, w)
    y2, _, m2, r2 = D.dprc_layernorm(x, w, stats=False)
    assert m2 is None and r2 is None and torch.equal(y, y2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        y3, _, _, _ = D.dprc_layernorm(x, w)
        dx3, _, dw3, db3 = D.dprc_layernorm_backward(x, x, w, *D.dprc_layernorm(x, w)[2:])
    st.synchronize()
    assert torch.equal(y, y3)
    dx, _, dw, db = D.dprc_layernorm_backward(x, x, w, *D.dprc_layernorm(x, w)[2:])
    assert torch.equal(dx, dx3) and torch.equal(dw, dw3) and torch.equal(db, db3)


# ---- backward -------------------------------------------------------------------------------------

def check_backward(D, dy, s, w, kind, ds, p, eps=EPS, **kw):
    dtype = "bf16" if s.dtype == torch.bfloat16 else "f32"
    rms = kind == D.RMSNORM
    B, T, n = s.shape
    _, m64, r64 = J.norm(s, eps=eps, rms=rms)
    mean = None if rms else torch.from_numpy(m64).float().cuda()
    rstd = torch.from_numpy(r64).float().cuda()
    dx, dh, dw, db = D.dprc_layernorm_backward(dy, s, w, mean, rstd, kind=kind, ds=ds, p=p, seed=SEED, site_id=SITE, **kw)
    rdx, rdw, rdb = J.norm_backward(dy, s, w, mean, rstd, ds=ds)
    K = max(64, n / 64)
    s64, dy64, r3 = as_f64(s), as_f64(dy), as_f64(rstd).reshape(B, T, 1)
    mu = np.zeros_like(r3) if rms else as_f64(mean).reshape(B, T, 1)
    xh = (s64 - mu) * r3
    exh = 2 * U * np.abs(xh) + U * r3 * np.abs(s64 - mu)
    g = dy64 * (np.ones(n) if w is None else as_f64(w))
    ag, agx = np.abs(g).mean(-1, keepdims=True), np.abs(g * xh).mean(-1, keepdims=True)
    sg = np.zeros_like(ag) if rms else (K + 4) * U * ag
    sgx = (K + 6) * U * agx + (np.abs(g) * exh).mean(-1, keepdims=True)
    tol = r3 * (8 * U * (np.abs(g) + ag + np.abs(xh) * agx) + sg + np.abs(xh) * sgx + exh * agx) + 4 * U * np.abs(rdx)
    if ds is not None:
        tol += 2 * U * np.abs(as_f64(ds))
    within(dx, rdx, tol + R[dtype] * np.abs(rdx))
    if p > 0:
        f = J.dropout_factors(SEED, SITE, B * T, n, p).reshape(B, T, n)
        rdh = rdx * f
        within(dh, rdh, f * tol + (2 * U + R[dtype]) * np.abs(rdh))
        assert torch.equal(dh == 0, torch.from_numpy(f == 0).cuda() | (dx == 0))
    else:
        assert dh is None
    if dw is not None:
        within(dw, rdw, ((T + 10) * U * np.abs(dy64 * xh) + np.abs(dy64) * exh).sum(1))
    if db is not None:
        within(db, rdb, (T + 8) * U * np.abs(dy64).sum(1))
    return dx, dh, dw, db


@pytest.mark.parametrize("kind", ["LAYERNORM", "RMSNORM"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 31, 63, 64, 65, 111, 128, 200, 256, 257, 500, 512, 513, 1000, 1024, 1025,
                               1111, 1536, 1537, 2048, 2049, 4000, 4096, 4097, 8192, 8200, 16384, 16391, 32768, 32776,
                               40003])
def test_backward_widths(D, n, dtype, kind):
    B, T = (2, 19) if n <= 4096 else (1, 3)
    k = getattr(D, kind)
    dy, s, ds = rows(B, T, n, dtype, n), rows(B, T, n, dtype, n + 1, shift=0.3), rows(B, T, n, dtype, n + 2)
    w = vec(n, dtype, n + 3, shift=1.0)
    check_backward(D, dy, s, w, k, ds, 0.1)
    check_backward(D, dy, s, w, k, None, 0.0)


@pytest.mark.parametrize("kind", ["LAYERNORM", "RMSNORM"])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("B,T,n,pad", [(1, 1, 64, 0), (1, 1, 2048, 0), (64, 1, 2048, 3), (1, 700, 64, 0), (5, 333, 111, 1),
                                       (2, 100, 2048, 8), (300, 3, 1111, 5), (1, 2000, 200, 0), (3, 257, 520, 0)])
def test_backward_forms(D, B, T, n, pad, dtype, wdtype, kind):
    k = getattr(D, kind)
    dy, s, ds = rows(B, T, n, dtype, 1, pad), rows(B, T, n, dtype, 2, pad, shift=0.5), rows(B, T, n, dtype, 3, pad)
    w = vec(n, wdtype, 4, shift=1.0)
    for d in (None, ds):
        for p in (0.0, 0.25):
            check_backward(D, dy, s, w, k, d, p)
    check_backward(D, dy, s, None, k, ds, 0.5)
    check_backward(D, dy, s, w, k, ds, 0.0, weight_grad=False, bias_grad=False)
    check_backward(D, dy, s, w, k, ds, 0.0, bias_grad=False)
    check_backward(D, dy, s, w, k, ds, 0.1, weight_grad=False)


def test_backward_outputs_one_by_one(D):
    # each output may be left out: the others stay what they are
    B, T, n = 3, 70, 200
    dy, s, ds, w = rows(B, T, n, "bf16", 1), rows(B, T, n, "bf16", 2), rows(B, T, n, "bf16", 3), vec(n, "bf16", 4, shift=1.0)
    _, _, mean, rstd = D.dprc_layernorm(s, w)
    full = D.dprc_layernorm_backward(dy, s, w, mean, rstd, ds=ds, p=0.2, seed=SEED, site_id=SITE)
    import ctypes
    L = D._ln(dy, D.LAYERNORM, w, None, 0.0, 0.2, SEED, SITE)
    need = D.lib().dprc_layernorm_backward_workspace(ctypes.byref(L))
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    for keep in range(1, 16):
        outs = [torch.full_like(t, 7.0) for t in full]
        ptr = [o.data_ptr() if keep >> j & 1 else None for j, o in enumerate(outs)]
        st = D.lib().dprc_layernorm_backward(ctypes.byref(L), dy.data_ptr(), n, s.data_ptr(), n, mean.data_ptr(),
                                             rstd.data_ptr(), ds.data_ptr(), n, ptr[0], n, ptr[1], n, ptr[2], ptr[3],
                                             n, ws.data_ptr(), need, D._stream(dy.device))
        assert st == D.SUCCESS
        for j in range(4):
            assert torch.equal(outs[j], full[j] if keep >> j & 1 else torch.full_like(full[j], 7.0)), (keep, j)


def test_backward_into_one_buffer_and_in_place(D):
    B, T, n = 3, 130, 200
    G = torch.full((B, 3 * n + 5), 7.0, device="cuda")
    for dtype in ("bf16", "f32"):
        dy, s, ds, w = rows(B, T, n, dtype, 1), rows(B, T, n, dtype, 2), rows(B, T, n, dtype, 3), vec(n, dtype, 4, shift=1.0)
        _, _, mean, rstd = D.dprc_layernorm(s, w)
        call = lambda dy, ds, **kw: D.dprc_layernorm_backward(dy, s, w, mean, rstd, ds=ds, p=0.1, seed=SEED, site_id=SITE, **kw)
        dx, dh, dw, db = call(dy, ds)
        call(dy, ds, dw=G[:, 3:3 + n], db=G[:, n + 4:2 * n + 4])
        assert torch.equal(G[:, 3:3 + n], dw) and torch.equal(G[:, n + 4:2 * n + 4], db)
        assert (G[:, :3] == 7.0).all() and (G[:, n + 3] == 7.0).all() and (G[:, 2 * n + 4:] == 7.0).all()
        a, b = dy.clone(), ds.clone()
        call(a, b, dx=b, dh=a)
        assert torch.equal(a, dh) and torch.equal(b, dx)
        a = s.clone()
        D.dprc_layernorm_backward(dy, a, w, mean, rstd, ds=ds, p=0.1, seed=SEED, site_id=SITE, dx=a)
        assert torch.equal(a, dx)


def test_backward_against_differences(D):
    # the library's own forward pass in fp32, differenced in directions of x, res, weight and bias
    B, T, n, p, h = 2, 40, 96, 0.2, 2.0 ** -6
    x, z, dy, q = (rows(B, T, n, "f32", j).double() for j in range(4))
    w, b = vec(n, "f32", 5, shift=1.0).double(), vec(n, "f32", 6).double()
    for kind in (D.LAYERNORM, D.RMSNORM):
        def outs(x, z, w, b):
            y, s, _, _ = D.dprc_layernorm(x.float(), w.float(), b.float(), kind=kind, res=z.float(), p=p, seed=SEED, site_id=SITE)
            return y.double(), s.double()
        _, s, mean, rstd = D.dprc_layernorm(x.float(), w.float(), b.float(), kind=kind, res=z.float(), p=p, seed=SEED, site_id=SITE)
        dx, dh, dw, db = D.dprc_layernorm_backward(dy.float(), s, w.float(), mean, rstd, kind=kind, ds=q.float(), p=p,
                                                   seed=SEED, site_id=SITE)
        for j, grad in enumerate((dh, dx, dw.sum(0), db.sum(0))):
            args = [x, z, w, b]
            g = torch.Generator().manual_seed(100 + j)
            v = torch.randn(args[j].shape, generator=g, dtype=torch.float64).cuda()
            # fourth-order differences, step h: the error h^4 y^(5) / 30 and 2 u |y| / h per element
            d = [0.0] * 4
            for i, k in enumerate((-2, -1, 1, 2)):
                args[j] = (x, z, w, b)[j] + k * h * v
                y, ss = outs(*args)
                d[i] = (y * dy).sum() + (ss * q).sum()
            num = ((d[0] - d[3]) + 8 * (d[2] - d[1])) / (12 * h)
            ana = (grad.double() * v).sum()
            scale = (grad.double().abs() * v.abs()).sum()
            assert abs(num - ana) <= 1e-3 * scale, (kind, j, float(num), float(ana), float(scale))


def test_sample_gradients_stay_apart(D):
    # zeroing one sample's dy changes that sample's rows alone
    B, T, n = 4, 300, 256
    dy, s = rows(B, T, n, "bf16", 1), rows(B, T, n, "bf16", 2)
    _, _, mean, rstd = D.dprc_layernorm(s)
    _, _, dw, db = D.dprc_layernorm_backward(dy, s, None, mean, rstd)
    z = dy.clone()
    z[2] = 0
    dx2, _, dw2, db2 = D.dprc_layernorm_backward(z, s, None, mean, rstd)
    assert (dw2[2] == 0).all() and (db2[2] == 0).all() and (dx2[2] == 0).all()
    for i in (0, 1, 3):
        assert torch.equal(dw[i], dw2[i]) and torch.equal(db[i], db2[i])


def test_same_call_same_bits(D):
    dy, s = rows(2, 900, 520, "bf16", 1), rows(2, 900, 520, "bf16", 2)
    _, _, mean, rstd = D.dprc_layernorm(s)
    first = D.dprc_layernorm_backward(dy, s, None, mean, rstd, p=0.1, seed=1)
    G = torch.randn(9, 30000, device="cuda")
    n2, gr = D.dprc_norm_vectors(G), D.dprc_clip_accumulate_vectors(G, torch.rand(9, device="cuda").fill_(0.3))
    for _ in range(3):
        for a, b in zip(first, D.dprc_layernorm_backward(dy, s, None, mean, rstd, p=0.1, seed=1)):
            assert torch.equal(a, b)
        assert torch.equal(n2, D.dprc_norm_vectors(G))
        assert torch.equal(gr, D.dprc_clip_accumulate_vectors(G, torch.full((9,), 0.3, device="cuda")))


def test_offsets_past_32_bits(D):
    # rows 2^22 elements apart: the last ones start beyond 2^31 elements (bf16) or bytes from the first
    n, T, ld = 72, 600, 1 << 22
    big = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((1, T, n), (T * ld, ld, 1))
    src = rows(1, T, n, "bf16", 1)
    far.copy_(src)
    assert torch.equal(D.dprc_dropout(far, 0.1, SEED, SITE), D.dprc_dropout(src, 0.1, SEED, SITE))
    y, s, mean, rstd = D.dprc_layernorm(src, p=0.1, seed=SEED, site_id=SITE)
    yf, sf, mf, rf = D.dprc_layernorm(far, p=0.1, seed=SEED, site_id=SITE)
    assert torch.equal(y, yf) and torch.equal(s, sf) and torch.equal(mean, mf)
    for a, b in zip(D.dprc_layernorm_backward(src, s, None, mean, rstd, p=0.1),
                    D.dprc_layernorm_backward(far, s, None, mean, rstd, p=0.1)):
        assert torch.equal(a, b)
    D.dprc_dropout(src, 0.1, SEED, SITE, out=far)
    assert torch.equal(far, D.dprc_dropout(src, 0.1, SEED, SITE))


# ---- per-sample vectors ---------------------------------------------------------------------------

@pytest.mark.parametrize("B,n,pad", [(1, 1, 0), (2, 3, 1), (8, 200, 0), (1, 100000, 0), (300, 70, 3), (8, 4097, 1),
                                     (33, 20000, 4), (2000, 5, 0), (5, 67584, 0)])
def test_vectors(D, B, n, pad):
    g = torch.Generator().manual_seed(B + n)
    G = torch.full((B, n + pad), float("nan"))
    G[:, :n] = torch.randn(B, n, generator=g) * torch.exp(torch.randn(B, 1, generator=g))
    G = G.cuda()[:, :n]
    c = (1.5 * torch.rand(B, generator=g) - 0.3).clamp(0, 1).cuda()
    n2, gr = D.dprc_norm_vectors(G), D.dprc_clip_accumulate_vectors(G, c)
    r2, rg = J.norm_vectors(G), J.clip_accumulate_vectors(G, c)
    within(n2, r2, 2 * U * r2)
    mag = (as_f64(c)[:, None] * np.abs(as_f64(G))).sum(0)
    within(gr, rg, (B + 2) * U * mag)
    base2, baseg = torch.rand(B, generator=g).cuda(), torch.randn(n, generator=g).cuda()
    got2 = D.dprc_norm_vectors(G, n2=base2.clone(), accumulate=True)
    gotg = D.dprc_clip_accumulate_vectors(G, c, grad=baseg.clone(), accumulate=True)
    within(got2, as_f64(base2) + r2, 3 * U * (as_f64(base2) + r2))
    within(gotg, as_f64(baseg) + rg, (B + 3) * U * (mag + np.abs(as_f64(baseg))))


def test_dropped_samples_have_no_part(D):
    G = torch.randn(6, 3001, device="cuda")
    c = torch.tensor([0.5, 0.0, 1.0, 0.0, 0.25, 0.0], device="cuda")
    ref = D.dprc_clip_accumulate_vectors(G, c)
    G[1], G[3, 5], G[5] = float("nan"), float("inf"), -float("inf")
    assert torch.equal(D.dprc_clip_accumulate_vectors(G, c), ref)
    n2 = D.dprc_norm_vectors(G)
    assert torch.isfinite(n2[[0, 2, 4]]).all() and not torch.isfinite(n2[[1, 3, 5]]).any()
    assert torch.equal(D.dprc_clip_accumulate_vectors(G, torch.zeros(6, device="cuda")), torch.zeros(3001, device="cuda"))
    assert torch.equal(D.dprc_clip_scale(n2, 1.0)[[1, 3, 5]], torch.zeros(3, device="cuda"))


# ---- graphs ------------------------------------------------------------------------------------------

def test_graph_replays(D):
    B, T, n = 2, 300, 520
    x, z, dy, w = rows(B, T, n, "bf16", 1), rows(B, T, n, "bf16", 2), rows(B, T, n, "bf16", 3), vec(n, "bf16", 4, shift=1.0)
    c = torch.rand(B, device="cuda")
    G = torch.empty(B, 2 * n, device="cuda")

    def step():
        y, s, mean, rstd = D.dprc_layernorm(x, w, res=z, p=0.1, seed=SEED, site_id=SITE)
        dx, dh, _, _ = D.dprc_layernorm_backward(dy, s, w, mean, rstd, ds=dy, p=0.1, seed=SEED, site_id=SITE,
                                                 dw=G[:, :n], db=G[:, n:])
        return y, s, dx, dh, D.dprc_norm_vectors(G), D.dprc_clip_accumulate_vectors(G, c), \
            D.dprc_dropout(x, 0.1, SEED, SITE)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(4):
        x.copy_(rows(B, T, n, "bf16", 10 + k))
        dy.copy_(rows(B, T, n, "bf16", 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), k


# ---- many short samples, rows of every remainder in place ---------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,n", [(700, 1, 5), (700, 5, 64), (1100, 3, 100), (520, 7, 300), (600, 2, 520), (1500, 1, 1024),
                                   (1030, 4, 1100), (2100, 9, 66)])
def test_many_short_samples(D, B, T, n, dtype):
    # more samples than workgroups, and samples of fewer tokens than a workgroup takes at a time
    dy, s, ds = rows(B, T, n, dtype, 1), rows(B, T, n, dtype, 2, shift=0.5), rows(B, T, n, dtype, 3)
    check_backward(D, dy, s, vec(n, dtype, 4, shift=1.0), D.LAYERNORM, ds, 0.25)
    check_backward(D, dy, s, None, D.RMSNORM, None, 0.0, bias_grad=False)


@pytest.mark.parametrize("B,T", [(1, 1000), (3, 777), (37, 61), (255, 40), (300, 33)])
@pytest.mark.parametrize("n", [40, 300])
def test_samples_cut_at_any_token(D, B, T, n):
    # the rows of all samples are dealt out evenly, so workgroups end and begin within samples
    dy, s = rows(B, T, n, "f32", 1), rows(B, T, n, "f32", 2, shift=0.5)
    check_backward(D, dy, s, vec(n, "f32", 4, shift=1.0), D.LAYERNORM, None, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [9, 67, 130, 257, 1111, 2047, 4099, 8190, 9001])
def test_in_place_at_every_remainder(D, n, dtype):
    # a row's last piece overlaps others' columns: in place it still sees the row as it was
    B, T = 3, 45
    x, z, w = rows(B, T, n, dtype, 1), rows(B, T, n, dtype, 2), vec(n, dtype, 3, shift=1.0)
    y, s, mean, rstd = D.dprc_layernorm(x, w, res=z, p=0.1, seed=SEED, site_id=SITE)
    a, b = x.clone(), z.clone()
    D.dprc_layernorm(a, w, res=b, p=0.1, seed=SEED, site_id=SITE, y=a, s=b)
    assert torch.equal(a, y) and torch.equal(b, s)
    dy, ds = rows(B, T, n, dtype, 4), rows(B, T, n, dtype, 5)
    call = lambda dy, s, ds, **kw: D.dprc_layernorm_backward(dy, s, w, mean, rstd, ds=ds, p=0.1, seed=SEED, site_id=SITE, **kw)
    dx, dh, dw, db = call(dy, s, ds)
    for which in (0, 1, 2):
        ins = [dy.clone(), s.clone(), ds.clone()]
        got = call(*ins, dx=ins[which], dh=ins[(which + 1) % 3])
        for u, v in zip(got, (dx, dh, dw, db)):
            assert torch.equal(u, v), which
    a = x.clone()
    assert torch.equal(D.dprc_dropout(a, 0.1, SEED, SITE, res=z, out=a), D.dprc_dropout(x, 0.1, SEED, SITE, res=z))
