"""Rotary positions against the 64-bit oracle.

Tolerance, u = 2^-24 and r = 2^-8 for bf16 results (0 for fp32): the angle is exact to 2^-40 of a turn, its fraction is
rounded once (pi u of a radian), sine and cosine are off by 2 ulp (2 u), their product with the scale, the two
products and their sum by u each: 10 u scale (|a| + |b|), and r of the result.
"""

import numpy as np
import pytest
import torch

from oracle import head as O
from oracle.estimators import as_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
R = {"bf16": 2.0 ** -8, "f32": 0.0}


@pytest.fixture(scope="module")
def D():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc
    dprc.lib()
    return dprc


def freqs(r, base=500000.0):
    return torch.tensor(base, dtype=torch.float64) ** (-torch.arange(r, dtype=torch.float64) / r)


def make(B, T, H, Dh, dtype, seed=0):
    return torch.randn(B, T, H, Dh, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).cuda()


def check(got, x, f, pos, out, scale=1.0, interleaved=False, inverse=False):
    xn, r = as_f64(x), len(f)
    ref = O.rotary(xn, f.cpu().numpy(), pos, scale, interleaved, inverse)
    ia = np.arange(r) * 2 if interleaved else np.arange(r)
    ib = ia + 1 if interleaved else ia + r
    tol = R[out] * np.abs(ref)
    both = 10 * U * scale * (np.abs(xn[..., ia]) + np.abs(xn[..., ib]))
    tol[..., ia] += both
    tol[..., ib] += both
    assert got.shape == x.shape and got.dtype == DT[out]
    bad = ~(np.abs(as_f64(got) - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("B,T,H,Dh,r", [(1, 1, 1, 2, 1), (2, 7, 3, 64, 32), (1, 130, 5, 80, 20), (3, 33, 2, 96, 13),
                                        (2, 5, 4, 129, 9), (64, 1, 8, 128, 64), (1, 9, 2, 256, 128), (2, 600, 40, 64, 32)])
def test_shapes(D, B, T, H, Dh, r, dtype, out, interleaved):
    x, f = make(B, T, H, Dh, dtype, seed=Dh), freqs(r).cuda()
    pos = torch.randint(-1000, 1_000_000, (B, T), generator=torch.Generator().manual_seed(r))
    kw = dict(interleaved=interleaved, out_dtype=DT[out])
    plain = np.broadcast_to(np.arange(T), (B, T))
    check(D.dprc_rotary(x, f, **kw), x, f, plain, out, interleaved=interleaved)
    check(D.dprc_rotary(x, f, start=77, heads_first=True, **kw), x, f, plain + 77, out, interleaved=interleaved)
    check(D.dprc_rotary(x, f, pos=pos.cuda(), scale=1.25, **kw), x, f, pos.numpy(), out, 1.25, interleaved)
    check(D.dprc_rotary(x, f, pos=pos.cuda(), inverse=True, **kw), x, f, pos.numpy(), out, 1.0, interleaved, True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Dh,r", [(3, 2, 8192, 4096), (2, 1, 1 << 20, 4096), (2, 1, 1 << 20, 1), (2, 1 << 16, 16, 8), (3, 1 << 16, 3, 1)])
def test_ends_of_the_ranges(D, T, H, Dh, r, dtype, interleaved):
    """The most pairs, the widest head, the most heads.  (The product and the reduction of an angle are off by about 2^-52
    of it: 2^-32 of a radian at a position of 10^6, far below the roundings to 32 bits.)"""
    x, f = make(1, T, H, Dh, dtype, seed=r), freqs(r).cuda()
    pos = torch.tensor([[1_000_000, 3, 77]])[:, :T]
    check(D.dprc_rotary(x, f, pos=pos.cuda(), interleaved=interleaved), x, f, pos.numpy(), dtype, interleaved=interleaved)
    want = D.dprc_rotary(x, f, start=5, inverse=True, interleaved=interleaved)
    check(want, x, f, 5 + np.arange(T)[None], dtype, interleaved=interleaved, inverse=True)
    if H > 2:                                            # as many in two tensors
        a, b = D.dprc_rotary([x[:, :, :-1], x[:, :, -1:]], f, start=5, inverse=True, interleaved=interleaved)
        assert torch.equal(torch.cat([a, b], 2), want)
    D.dprc_rotary(x, f, start=5, inverse=True, interleaved=interleaved, out=x)
    assert torch.equal(x, want)


def test_far_positions(D):
    """Angles of 2^40 radians and more."""
    x, f = make(1, 4, 2, 64, "f32"), freqs(32).cuda()
    pos = torch.tensor([[2 ** 31, 2 ** 33 + 1, 2 ** 20, 0]])
    # the angle's product and its reduction are off by 2^-52 of it: 2^33 2^-52 2 pi 2 of a radian more than elsewhere
    got, ref = as_f64(D.dprc_rotary(x, f, pos=pos.cuda())), O.rotary(as_f64(x), f.cpu().numpy(), pos.numpy())
    assert np.abs(got - ref).max() <= (10 * U + 2.0 ** -15) * 2 * np.abs(as_f64(x)).max()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_strided_tensors_and_in_place(D, dtype, interleaved):
    rows = make(2, 50, 4 + 2 * 3, 64, dtype)
    f = freqs(24).cuda()
    pos = np.broadcast_to(np.arange(50), (2, 50))
    q, k = rows[:, :, :4], rows[:, :, 4:7]
    before = rows.clone()
    a, b = D.dprc_rotary([q, k], f, interleaved=interleaved)
    assert torch.equal(rows, before)
    check(a, q, f, pos, dtype, interleaved=interleaved)
    check(b, k, f, pos, dtype, interleaved=interleaved)
    turned = q.transpose(1, 2).contiguous().transpose(1, 2)         # heads first
    assert torch.equal(D.dprc_rotary(turned, f, interleaved=interleaved), a)
    odd = torch.full((2, 50, 4, 67), 3.0, dtype=DT[dtype], device="cuda")
    D.dprc_rotary(q, f, interleaved=interleaved, out=odd[..., 1:65])
    assert torch.equal(odd[..., 1:65], a) and (odd[..., 0] == 3).all() and (odd[..., 65:] == 3).all()
    D.dprc_rotary([q, k], f, interleaved=interleaved, out=[q, k])   # in place
    assert torch.equal(q, a) and torch.equal(k, b) and torch.equal(rows[:, :, 7:], before[:, :, 7:])


def test_four_tensors_and_one_too_many(D):
    f = freqs(8).cuda()
    xs = [make(1, 3, h, 16, "f32", seed=h) for h in (1, 2, 3, 5)]
    for y, x in zip(D.dprc_rotary(xs, f), xs):
        check(y, x, f, np.arange(3)[None], "f32")
    with pytest.raises(RuntimeError):
        D.dprc_rotary(xs + xs[:1], f)


def test_inverse_is_the_transpose(D):
    """<rotary(x), y> = <x, inverse(y)>, and at scale 1 the inverse undoes the turn."""
    x, y, f = make(2, 40, 4, 64, "f32", 1), make(2, 40, 4, 64, "f32", 2), freqs(20).cuda()
    a = (D.dprc_rotary(x, f, scale=1.3).double() * y.double()).sum().item()
    b = (x.double() * D.dprc_rotary(y, f, scale=1.3, inverse=True).double()).sum().item()
    mag = 1.3 * 2 * (x.abs().double() * y.abs().double()).sum().item()
    assert abs(a - b) <= 20 * U * 3 * mag
    back = D.dprc_rotary(D.dprc_rotary(x, f), f, inverse=True)
    assert (back - x).abs().max() <= 40 * U * 4 * x.abs().max()


def test_large_strides(D):
    """Heads more than 2^31 elements apart."""
    big = torch.empty(2 ** 31 + 128, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((1, 2, 2, 32), (0, 32, 2 ** 31 + 32, 1))
    x.copy_(make(1, 2, 2, 32, "bf16"))
    f = freqs(16).cuda()
    check(D.dprc_rotary(x, f), x, f, np.arange(2)[None], "bf16")
    y = D.dprc_rotary(x, f)
    D.dprc_rotary(x, f, out=x)
    assert torch.equal(x, y)


def test_captured(D):
    q, k, f = make(2, 30, 4, 64, "bf16"), make(2, 30, 2, 64, "bf16", 1), freqs(32).cuda()
    pos = torch.arange(60, device="cuda").view(2, 30)
    graph = torch.cuda.CUDAGraph()
    D.dprc_rotary([q, k], f, pos=pos)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a, b = D.dprc_rotary([q, k], f, pos=pos)
    for step in range(3):
        pos.add_(1000)
        q.mul_(1.5)
        graph.replay()
        got = a.clone(), b.clone()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, D.dprc_rotary([q, k], f, pos=pos)))
