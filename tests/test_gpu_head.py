"""The output head's cross entropy and its gradients against the 64-bit oracle.

Tolerances, with u = 2^-24 and r = 2^-8 for bf16 heads (0 for fp32):

* a logit is a chain of at most d fp32 sums of exact (bf16) or once rounded products: off by (d + 1) u times the
  sum of its terms' magnitudes; delta_t is the largest of a token;
* exp(l - c) is taken as 2^(l log2 e - c log2 e): the product with log2 e, the two roundings of the
  difference and of log2 e itself are off by 4 u (|l| + |c|) at most in the exponent, 2^x by 4 u of itself,
  and what lies below the smallest normal number may become zero: 2^-126 for p and for E each;
* lse: the sum of V positive terms in chains of at most 160 + V / 128 roundings, the logarithm and its
  sum with the maximum 4 u of their magnitudes: delta + 4 u (|top| + max|l|) + (170 + V / 128) u + 4 u |lse|;
* loss: that, delta again for the target's logit, and u of the difference's terms;
* E: |g| p times what the exponent is off by, 8 u |E| for the products (of the target's entry: 4 u |g| more for
  the difference), and r |E|;
* dh, dW: E's own error through the product, chains of at most V (N) sums and 64 planes: (V + 64) u times the
  terms' magnitudes, and r of the result.
"""

import numpy as np
import pytest
import torch

from oracle import estimators as est
from oracle import head as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
R = {"bf16": 2.0 ** -8, "f32": 0.0}
f64 = est.as_f64


@pytest.fixture(scope="module")
def D():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc
    dprc.lib()
    return dprc


def make(B, T, d, V, dtype, seed=0, pad=0, wpad=0, scale=1.0, ignored="some"):
    """h, W, target, g; what lies between the rows is NaN, and so are the rows without a target."""
    gen = torch.Generator().manual_seed(seed)
    W = torch.full((V, d + wpad), float("nan"))
    W[:, :d] = torch.randn(V, d, generator=gen) * (scale / d ** 0.5)
    W = W.to(DT[dtype]).cuda()[:, :d]
    target = torch.randint(0, V, (B, T), generator=gen)
    h = torch.full((B, T, d + pad), float("nan"))
    h[..., :d] = torch.randn(B, T, d, generator=gen) + 4.0 * torch.rand(B, T, 1, generator=gen) * W.cpu()[target].float()
    if ignored == "some":
        target[torch.rand(B, T, generator=gen) < 0.2] = -100
    elif ignored == "all":
        target[:] = -1
    g = torch.randn(B, T, generator=gen) / T
    return h.to(DT[dtype]).cuda()[..., :d], W, target.cuda(), g.cuda()


def spoil(h, target, g):
    """NaN and infinity where nothing has a loss."""
    h, g = h.clone(), g.clone()
    h[target < 0] = float("nan")
    g[target < 0] = float("inf")
    return h, g


def delta(h, W):
    return (h.shape[-1] + 1) * U * (np.abs(h) @ np.abs(W).T).max(-1)


def exponent(h, W, lse):
    return delta(h, W) + 4 * U * (np.abs(h @ W.T).max(-1) + np.abs(lse))


def within(got, ref, tol, name=""):
    got = f64(got)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), got[bad][:4], ref[bad][:4], np.broadcast_to(tol, ref.shape)[bad][:4])


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 2), (2, 3, 5, 7), (1, 1, 64, 300), (2, 37, 72, 257), (3, 50, 136, 1009), (64, 1, 96, 1500),
          (65, 1, 200, 513), (1, 300, 129, 777), (2, 130, 320, 2050), (1, 257, 1030, 260)]


def check_loss(D, h, W, target):
    loss, lse = D.dprc_head_loss(h, W, target)
    hn, Wn, tn = f64(h), f64(W), target.cpu().numpy()
    rl, rz = O.loss(hn, Wn, tn)
    big = np.abs(hn @ Wn.T).max(-1)
    tz = delta(hn, Wn) + 8 * U * big + (170 + W.shape[0] / 128) * U + 4 * U * np.abs(rz)
    within(lse, rz, tz, "lse")
    within(loss, rl, np.where(tn < 0, 0.0, tz + delta(hn, Wn) + 2 * U * (np.abs(rz) + big)), "loss")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,d,V", SHAPES)
def test_loss(D, B, T, d, V, dtype):
    h, W, target, _ = make(B, T, d, V, dtype, seed=V)
    check_loss(D, h, W, target)


def check_backward(D, h, W, target, g, dtype, **kw):
    lse = D.dprc_head_loss(h, W, target)[1]
    hn, Wn, tn, zn, gn = f64(h), f64(W), target.cpu().numpy(), f64(lse), f64(g)
    E = O.errors(hn, Wn, tn, zn, gn)
    kept = (tn >= 0)[..., None]
    p = np.where(kept, np.exp(hn @ Wn.T - zn[..., None]), 0.0)
    ga = np.where(kept, np.abs(gn)[..., None], 0.0)
    tE = ga * p * (exponent(hn, Wn, zn)[..., None] + 8 * U) + 8 * U * np.abs(E) + R[dtype] * np.abs(E) + (1 + ga) * 2.0 ** -126
    np.put_along_axis(tE, np.maximum(tn, 0)[..., None], np.take_along_axis(tE + 4 * U * ga, np.maximum(tn, 0)[..., None], -1), -1)
    tE = np.where(kept, tE, 0.0)
    hs, gs = spoil(h, target, g)
    within(D.dprc_head_errors(hs, W, target, lse, gs), E, tE, "E")
    dh, dW = D.dprc_head_backward(hs, W, target, lse, gs, **kw)
    V, N = W.shape[0], h.shape[0] * h.shape[1]
    ref = E @ Wn
    within(dh, ref, tE @ np.abs(Wn) + (V + 64) * U * (np.abs(E) + tE) @ np.abs(Wn) + R[dtype] * 1.01 * np.abs(ref)
           + R[dtype] * tE @ np.abs(Wn), "dh")
    Ef, tf, hf = E.reshape(N, V), tE.reshape(N, V), np.where(kept, hn, 0.0).reshape(N, -1)
    ref = Ef.T @ hf
    own = tf.T @ np.abs(hf)
    within(dW, ref, own * (1 + R[dtype]) + (N + 64) * U * (np.abs(Ef) + tf).T @ np.abs(hf) + R[dtype] * 1.01 * np.abs(ref), "dW")
    return lse, E


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,d,V", SHAPES)
def test_backward(D, B, T, d, V, dtype):
    h, W, target, g = make(B, T, d, V, dtype, seed=V + 1)
    check_backward(D, h, W, target, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V,wpad", [(150, 136, 1009, 0), (40, 72, 900, 3), (900, 264, 3000, 0), (700, 520, 12000, 1)])
def test_gradients_alone(D, T, d, V, wpad, dtype):
    """dh and dW by themselves are those of the call for both."""
    h, W, target, g = make(2, T, d, V, dtype, seed=T, wpad=wpad)
    lse = D.dprc_head_loss(h, W, target)[1]
    dh, dW = D.dprc_head_backward(h, W, target, lse, g)
    assert torch.equal(D.dprc_head_backward(h, W, target, lse, g, weight_grad=False)[0], dh)
    assert torch.equal(D.dprc_head_backward(h, W, target, lse, g, hidden_grad=False)[1], dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,wpad,d", [(3, 0, 128), (8, 8, 128), (0, 5, 64), (1, 1, 131), (0, 0, 131), (4, 4, 132)])
def test_strides(D, pad, wpad, d, dtype):
    h, W, target, g = make(2, 90, d, 600, dtype, seed=pad, pad=pad, wpad=wpad)
    check_backward(D, h, W, target, g, dtype)
    base = D.dprc_head_loss(h.contiguous(), W.contiguous(), target)
    got = D.dprc_head_loss(h, W, target)
    for x, y in zip(base, got):
        torch.testing.assert_close(x, y, rtol=1e-6, atol=1e-6, equal_nan=True)
    # results into rows of their own, what lies between them left alone
    out = torch.full((2, 90, d + 5), 7.0, dtype=h.dtype, device="cuda")
    wide = torch.full((600, d + 3), 7.0, dtype=h.dtype, device="cuda")
    dh, dW = D.dprc_head_backward(h, W, target, base[1], g, dh=out[..., :d], dW=wide[:, :d])
    r = D.dprc_head_backward(h, W, target, base[1], g)
    assert torch.equal(dh, r[0]) and torch.equal(dW, r[1])
    assert (out[..., d:] == 7).all() and (wide[:, d:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,piece", [(20000, 8192), (16384, 8192), (16400, 16384), (8193, 8192), (17001, 0)])
def test_pieces(D, V, piece, dtype):
    h, W, target, g = make(2, 35, 48, V, dtype, seed=V)
    check_backward(D, h, W, target, g, dtype, piece=piece)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V,wpad", [(16, 1544, 300, 0), (33, 1030, 1000, 2), (70, 2050, 600, 2), (100, 776, 17000, 0), (40, 1000, 17000, 0),
                                        (32, 776, 17000, 1), (200, 1544, 300, 0)])
def test_long_contractions_of_few_tiles(D, T, d, V, wpad, dtype):
    """Slabs three ahead, contractions over the waves, narrow tiles, and W off the boundaries for each."""
    h, W, target, g = make(1, T, d, V, dtype, seed=T + d, wpad=wpad)
    check_loss(D, h, W, target)
    check_backward(D, h, W, target, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,d,V,wpad", [(1, 32, 776, 17000, 0), (1, 1, 132, 16388, 0), (31, 1, 136, 16385, 0), (7, 1, 131, 16400, 0)])
def test_few_tokens_of_a_large_vocabulary(D, B, T, d, V, wpad, dtype):
    """One column of narrow tiles, W in whole pieces straight to LDS or off its boundaries, a last tile of few rows."""
    h, W, target, g = make(B, T, d, V, dtype, seed=V, wpad=wpad)
    check_loss(D, h, W, target)
    check_backward(D, h, W, target, g, dtype)


@pytest.mark.parametrize("T,V", [(70, 66565), (700, 65700)])
def test_rows_past_whole_rounds_of_tiles(D, T, V):
    """Rounds of 256 tiles and a few more, whose rows of W are products of their own (dW's for 70 tokens; the logits' and
    dW's, split and rounded, for 700), with targets on both sides of the border and the largest logits past it."""
    h, W, target, g = make(1, T, 48, V, "bf16", seed=T)
    W[65500:] *= 3
    target[0, :6] = torch.tensor([65535, 65536, 65537, V - 1, 65535, 0], device="cuda")
    check_loss(D, h, W, target)
    check_backward(D, h, W, target, g, "bf16")


@pytest.mark.parametrize("B,T,d,V,wpad,piece", [(1, 1, 64, 300, 0, 0), (2, 77, 72, 1000, 0, 0), (2, 77, 72, 1000, 3, 0),
                                                (1, 700, 264, 20000, 0, 8192), (1, 300, 136, 9000, 0, 0), (4, 600, 520, 600, 0, 0)])
def test_the_targets_entry_enters_to_16_bits(D, B, T, d, V, wpad, piece):
    """bf16: of the target's entry of E no more is lost than 2^-17 (the second half of its split is rounded to bf16: 2^-8 of
    at most 2^-8 of it, halved), where the others are off by r: with one g for all tokens whose rounding is the worst
    there is, dh and dW are off by the rounding of the result and the others' share."""
    h, W, target, _ = make(B, T, d, V, "bf16", seed=V, wpad=wpad)
    target[0, T // 2:] = int(target[0, 0])                  # one target many times over
    g = torch.full((B, T), 1.0 + 2.0 ** -8, device="cuda")
    lse = D.dprc_head_loss(h, W, target)[1]
    hn, Wn, tn, zn = f64(h), f64(W), target.cpu().numpy(), f64(lse)
    E = O.errors(hn, Wn, tn, zn, f64(g))
    kept = (tn >= 0)[..., None]
    tE = R["bf16"] * np.abs(E)
    at = np.maximum(tn, 0)[..., None]
    np.put_along_axis(tE, at, 2.0 ** -17 * np.take_along_axis(np.abs(E), at, -1), -1)
    tE = np.where(kept, tE + 2 * np.where(kept, np.exp(hn @ Wn.T - zn[..., None]), 0) * (exponent(hn, Wn, zn)[..., None] + 8 * U)
                  + 16 * U * np.abs(E), 0.0)
    dh, dW = D.dprc_head_backward(h, W, target, lse, g, piece=piece)
    ref = E @ Wn
    within(dh, ref, (1 + R["bf16"]) * tE @ np.abs(Wn) + (V + 64) * U * np.abs(E) @ np.abs(Wn) + R["bf16"] * np.abs(ref), "dh")
    Ef, tf, hf = E.reshape(B * T, V), tE.reshape(B * T, V), np.where(kept, hn, 0.0).reshape(B * T, d)
    ref = Ef.T @ hf
    within(dW, ref, (1 + R["bf16"]) * tf.T @ np.abs(hf) + (B * T + 64) * U * np.abs(Ef).T @ np.abs(hf) + R["bf16"] * np.abs(ref), "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_laid_out_in_pieces(D, dtype):
    """Rows of W off the 16-byte boundaries and enough tokens for a copy of them: as with aligned rows."""
    T, V, d = 1100, 9000, 131
    h, W, target, g = make(1, T, d, V, dtype, seed=12, wpad=3)
    check_backward(D, h, W, target, g, dtype, piece=8192)
    hz, Wz = (torch.nn.functional.pad(x, (0, 5)) for x in (h, W))
    for a, b in zip(D.dprc_head_loss(h, W, target), D.dprc_head_loss(hz, Wz, target)):
        torch.testing.assert_close(a, b, rtol=1e-6, atol=1e-6)
    # more than a piece of the forward pass: 2^28 bytes of W
    d, V = 4093, 37000 if dtype == "bf16" else 17000
    h, W, target, g = make(1, 1024, d, V, dtype, seed=13)
    hz, Wz = (torch.nn.functional.pad(x, (0, 3)) for x in (h, W))
    for a, b in zip(D.dprc_head_loss(h, W, target), D.dprc_head_loss(hz, Wz, target)):
        torch.testing.assert_close(a, b, rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(D, dtype):
    """Probabilities of 1 and of 0: logits of hundreds."""
    h, W, target, g = make(2, 70, 64, 500, dtype, seed=5, scale=300.0)
    check_backward(D, h, W, target, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_targets_at_all(D, dtype):
    h, W, target, g = make(2, 70, 64, 500, dtype, seed=5, ignored="all")
    loss, lse = D.dprc_head_loss(h, W, target)
    assert (loss == 0).all() and lse.isfinite().all()
    hs, gs = spoil(h, target, g)
    dh, dW, n2 = D.dprc_head_backward(hs, W, target, lse, gs, k=4)
    assert not dh.any() and not dW.any() and not n2.any()
    assert not D.dprc_head_clip_accumulate(hs, W, target, lse, gs, torch.ones(2, device="cuda")).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_past_the_vocabulary_and_infinite_logits(D, dtype):
    h, W, target, g = make(2, 70, 64, 500, dtype, seed=6, ignored="none")
    clean = D.dprc_head_loss(h, W, target)
    target[0, 3], target[1, 5] = 500, 2 ** 40
    loss, lse = D.dprc_head_loss(h, W, target)
    bad = torch.zeros_like(target, dtype=torch.bool)
    bad[0, 3] = bad[1, 5] = True
    assert torch.equal(loss.isnan(), bad) and torch.equal(lse.isnan(), bad)
    assert torch.equal(loss[~bad], clean[0][~bad])
    dh, _ = D.dprc_head_backward(h, W, target, lse, g)
    assert torch.equal(dh.isnan().all(-1), bad) and torch.equal(dh.isnan().any(-1), bad)
    # a row of the vocabulary at -infinity takes no part (all features of h positive)
    hp, Wi = h.abs(), W.clone()
    Wi[17] = float("-inf")
    some = torch.where(target == 17, 18, target).clamp(max=499)
    keep = torch.arange(500, device="cuda") != 17
    l1, z1 = D.dprc_head_loss(hp, Wi, some)
    l0, z0 = D.dprc_head_loss(hp, W[keep].contiguous(), some - (some > 17).long())
    torch.testing.assert_close(z1, z0, rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(l1, l0, rtol=1e-5, atol=1e-5)
    assert (D.dprc_head_errors(hp, Wi, some, z1, g)[..., 17] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 67])
def test_a_sample_whose_errors_are_not_finite_is_clipped_to_nothing(D, d, dtype):
    """The largest and the smallest target there are, an infinite weight of a loss: of other samples nothing changes, and with
    the factor that the estimates give the clipped sum is theirs."""
    B, T, V = 4, 70, 9001
    h, W, target, g = make(B, T, d, V, dtype, seed=d, ignored="none")
    target[0, 3], target[0, 66] = -2 ** 63, -1
    clean = target.clone()
    target[1, 5], target[2, 64] = 2 ** 63 - 1, V
    loss, lse = D.dprc_head_loss(h, W, target)
    l0, z0 = D.dprc_head_loss(h, W, clean)
    bad = target != clean
    assert torch.equal(loss.isnan(), bad) and torch.equal(lse.isnan(), bad) and loss[0, 3] == 0 and loss[0, 66] == 0
    assert torch.equal(loss[~bad], l0[~bad]) and torch.equal(lse[~bad], z0[~bad])
    dh, _, n2 = D.dprc_head_backward(h, W, target, lse, g, weight_grad=False, k=8, seed=3)
    r, _, m2 = D.dprc_head_backward(h, W, clean, z0, g, weight_grad=False, k=8, seed=3)
    assert torch.equal(dh[~bad], r[~bad]) and dh[bad].isnan().all()
    gi = g.clone()
    gi[3, 7] = float("inf")
    n2 = torch.cat([n2[:3], D.dprc_head_backward(h, W, clean, z0, gi, hidden_grad=False, weight_grad=False, k=8, seed=3)[2][3:]])
    assert torch.equal(n2[:1], m2[:1]) and not n2[1:].isfinite().any()
    c = D.dprc_clip_scale(n2, 0.5)
    assert c[0] > 0 and not c[1:].any()
    got = D.dprc_head_clip_accumulate(h, W, target, lse, gi, c)
    assert got.isfinite().all() and torch.equal(got, D.dprc_head_clip_accumulate(h, W, clean, z0, g, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("side", [0, 1, 2])
@pytest.mark.parametrize("probe,k", [(0, 16), (2, 8), (0, 33)])
def test_private(D, dtype, side, probe, k):
    """The estimates are those of the head's blocks as layers, the clipped gradient theirs side by side."""
    B, T, d, V = 3, 40, 72, 20001
    h, W, target, g = make(B, T, d, V, dtype, seed=side)
    lse = D.dprc_head_loss(h, W, target)[1]
    E = D.dprc_head_errors(h, W, target, lse, g)
    hs, gs = spoil(h, target, g)
    start = torch.rand(B, device="cuda")
    for piece in (8192, 16384, 0):
        dh, dW, n2 = D.dprc_head_backward(hs, W, target, lse, gs, hidden_grad=False, weight_grad=False, k=k, seed=11,
                                          layer_id=7, side=side, probe=probe, piece=piece)
        assert dh is None and dW is None
        ref = 0
        for b, v0 in enumerate(range(0, V, D.HEAD_BLOCK)):
            Ab = torch.where((target >= 0)[..., None], h, torch.zeros_like(h)).contiguous()
            ref = ref + D.dprc_norm_hutch([(Ab, E[..., v0:v0 + D.HEAD_BLOCK].contiguous(), 7 + b)], k, 11, side=side,
                                          probe=probe).double()
        np.testing.assert_allclose(f64(n2), f64(ref), rtol=1e-5)
        more = start.clone()
        D.dprc_head_backward(hs, W, target, lse, gs, k=k, seed=11, layer_id=7, side=side, probe=probe, piece=piece, n2=more,
                             accumulate=True)
        np.testing.assert_allclose(f64(more), f64(start) + f64(n2), rtol=1e-5)
        c = torch.tensor([0.5, 0.0, 1.0], device="cuda")
        grad = D.dprc_head_clip_accumulate(hs, W, target, lse, gs, c, piece=piece)
        En, hn, cn = f64(E), np.where((target >= 0).cpu().numpy()[..., None], f64(h), 0.0), f64(c)
        rg = est.clip_accumulate(hn, En, cn)
        mag = est.clip_accumulate(np.abs(hn), np.abs(En), cn)
        within(grad, rg, (B * T + 8) * U * mag, "grad")       # chains of B T sums, a rescaling for every sample
        wide = torch.full((d, V + 3), 2.0, device="cuda")
        D.dprc_head_clip_accumulate(hs, W, target, lse, gs, c, grad=wide[:, :V], accumulate=True, piece=piece)
        within(wide[:, :V], rg + 2.0, (B * T + 8) * U * mag + U * (np.abs(rg) + 2.0), "grad")
        assert (wide[:, V:] == 2).all()


def test_errors_of_columns(D):
    h, W, target, g = make(2, 40, 64, 3001, "bf16", seed=9)
    lse = D.dprc_head_loss(h, W, target)[1]
    E = D.dprc_head_errors(h, W, target, lse, g)
    buf = torch.full((2, 40, 1007), 5.0, dtype=torch.bfloat16, device="cuda")
    for v0, nv in ((0, 1), (3000, 1), (1234, 1001), (256, 512)):
        buf[:] = 5.0
        out = D.dprc_head_errors(h, W, target, lse, g, v0=v0, nv=nv, E=buf[..., 1:1 + nv])
        assert torch.equal(out, E[..., v0:v0 + nv])
        assert (buf[..., 0] == 5).all() and (buf[..., 1 + nv:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_is_that_of_differences(D, dtype):
    """sum g loss along a direction of h and of W against dh and dW (fp32 inputs; bf16 through its own loss)."""
    h, W, target, g = make(2, 20, 40, 300, dtype, seed=3)
    lse = D.dprc_head_loss(h, W, target)[1]
    dh, dW = D.dprc_head_backward(h, W, target, lse, g)
    hn, Wn, tn, gn = f64(h), f64(W), target.cpu().numpy(), f64(g)
    rng = np.random.default_rng(0)
    uh, uw, eps = rng.standard_normal(hn.shape), rng.standard_normal(Wn.shape), 1e-5
    f = lambda a: (gn * O.loss(hn + a * uh, Wn + a * uw, tn)[0]).sum()
    slope = (f(eps) - f(-eps)) / (2 * eps)
    terms = np.abs(f64(dh) * uh).sum() + np.abs(f64(dW) * uw).sum()
    # the difference's own error is of order eps^2; the gradients' that of the other tests
    assert abs((f64(dh) * uh).sum() + (f64(dW) * uw).sum() - slope) <= (2 * R[dtype] + 1e-5) * terms


def test_repeats_and_streams(D):
    """Two calls at once, on streams of their own with workspaces of their own, give what one gives."""
    h, W, target, g = make(2, 300, 128, 9000, "bf16", seed=4)
    lse = D.dprc_head_loss(h, W, target)[1]
    ref = D.dprc_head_backward(h, W, target, lse, g, k=8, seed=1)
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    out = []
    for st in s:
        with torch.cuda.stream(st):
            l, z = D.dprc_head_loss(h, W, target)
            out.append((z, *D.dprc_head_backward(h, W, target, z, g, k=8, seed=1)))
    torch.cuda.synchronize()
    for z, *rest in out:
        assert torch.equal(z, lse) and all(torch.equal(a, b) for a, b in zip(rest, ref))


@pytest.mark.parametrize("odd", [0, 1])
def test_strides_past_32_bits(D, odd):
    """Rows so far apart that offsets pass 2^32 bytes: what rows side by side give."""
    B, T, d, V = 2, 75, 64, 4500
    h, W, target, g = make(B, T, d, V, "bf16", seed=4)
    far = lambda rows, ld: torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)[:, :d]
    ld = (1 << 19) + 8 + odd
    ref_W = far(V, 72 + odd)                              # the same path: whole pieces, or rows off their boundaries
    ref_W.copy_(W)
    far_W, far_h = far(V, ld), far(B * T, 1 << 24).unflatten(0, (B, T))
    far_W.copy_(W)
    far_h.copy_(h)
    assert far_W.stride(0) * V * 2 > 1 << 32 and far_h.stride(1) * B * T * 2 > 1 << 32
    loss, lse = D.dprc_head_loss(h, ref_W, target)
    for got, want in zip(D.dprc_head_loss(far_h, far_W, target), (loss, lse)):
        assert torch.equal(got, want)
    want = D.dprc_head_backward(h, ref_W, target, lse, g, k=4, seed=1)
    dW, dh = far(V, ld), far(B * T, 1 << 24).unflatten(0, (B, T))
    for got, w in zip(D.dprc_head_backward(far_h, far_W, target, lse, g, k=4, seed=1, dh=dh, dW=dW), want):
        assert torch.equal(got, w)
    E = far(B * T, 1 << 24).unflatten(0, (B, T))
    assert torch.equal(D.dprc_head_errors(far_h, far_W, target, lse, g, v0=4400, nv=d, E=E),
                       D.dprc_head_errors(h, ref_W, target, lse, g, v0=4400, nv=d))


def test_captured(D):
    h, W, target, g = make(2, 100, 128, 9000, "bf16", seed=8)
    static = dict(h=h.clone(), g=g.clone(), target=target.clone())
    c = torch.tensor([0.5, 1.0], device="cuda")

    def step():
        loss, lse = D.dprc_head_loss(static["h"], W, static["target"])
        dh, dW, n2 = D.dprc_head_backward(static["h"], W, static["target"], lse, static["g"], k=8, seed=1)
        return loss, lse, dh, dW, n2, D.dprc_head_clip_accumulate(static["h"], W, static["target"], lse, static["g"], c)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (8, 21, 22):
        h2, _, t2, g2 = make(2, 100, 128, 9000, "bf16", seed=seed)
        for k, v in dict(h=h2, g=g2, target=t2).items():
            static[k].copy_(v)
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
