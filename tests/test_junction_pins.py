"""The oracle of dropout, norm and the norms' private gradients, against torch's own forms in
64 bits, differences, and the statistics a dropout mask has to have (no GPU)."""

import numpy as np
import pytest
import torch

from oracle import junction as J

SEED, SITE = 0x1234567890ABCDEF, 7


def _rows(B, T, n, seed):
    return np.random.default_rng(seed).standard_normal((B, T, n))


def test_dropout_bits_are_the_counter_generator():
    # the same block read word by word through the generator's own definition
    from oracle import philox
    rows, n = 3, 21
    bits = J.dropout_bits(SEED, SITE, rows, n)
    for r in range(rows):
        for c in range(n):
            words = philox.philox4x32_10(np.array([c // 8, r, SITE, 4]), philox._key(SEED))
            assert bits[r, c] == (int(words[(c % 8) // 2]) >> (16 * (c % 2))) & 0xFFFF
    assert np.array_equal(J.dropout_bits(SEED, SITE, 2, n, row0=1), bits[1:])


@pytest.mark.parametrize("p", [2.0 ** -16, 0.1, 0.5, 0.9])
def test_dropout_rate_and_mean(p):
    rows, n = 512, 1024
    f = J.dropout_factors(SEED, SITE, rows, n, p)
    q = np.floor(65536 * float(np.float32(p)) + 0.5) / 65536
    N = rows * n
    assert abs((f == 0).mean() - q) <= 5 * np.sqrt(q * (1 - q) / N)        # five standard deviations
    assert abs(f.mean() - 1.0) <= 5 * np.sqrt(q / (1 - q) / N)             # unbiased


def test_dropout_masks_are_independent_over_rows_columns_sites_and_seeds():
    f = (J.dropout_bits(SEED, SITE, 256, 512) < 32768) * 2.0 - 1.0
    N = f.size
    for other in ((J.dropout_bits(SEED, SITE + 1, 256, 512) < 32768) * 2.0 - 1.0,
                  (J.dropout_bits(SEED + 1, SITE, 256, 512) < 32768) * 2.0 - 1.0,
                  np.roll(f, 1, 0), np.roll(f, 1, 1), np.roll(f, 2, 1), np.roll(f, 8, 1)):
        assert abs((f * other).mean()) <= 5 / np.sqrt(N)


def test_dropout_edges():
    x = np.array([[[np.nan, np.inf, -np.inf, 3.0]]])
    assert np.array_equal(J.dropout(x, 0, 0, 1.0), np.zeros((1, 1, 4)))     # all dropped, whatever they were
    assert np.array_equal(J.dropout(x, 0, 0, 0.0)[0, 0, 1:], x[0, 0, 1:])   # none dropped
    assert np.array_equal(J.dropout(x, 0, 0, 1.0, res=x)[0, 0, 1:], x[0, 0, 1:])


@pytest.mark.parametrize("B,T,n", [(1, 1, 1), (2, 3, 5), (3, 4, 64)])
def test_layer_norm_is_torchs(B, T, n):
    s, dy = _rows(B, T, n, 1) + 0.3, _rows(B, T, n, 2)
    w, b = 1 + 0.1 * _rows(1, 1, n, 3)[0, 0], 0.1 * _rows(1, 1, n, 4)[0, 0]
    y, mean, rstd = J.norm(s, w, b, eps=1e-5)
    ts = torch.tensor(s, requires_grad=True)
    tw, tb = torch.tensor(w), torch.tensor(b)
    ty = torch.nn.functional.layer_norm(ts, (n,), tw, tb, eps=float(np.float32(1e-5)))
    assert np.allclose(y, ty.detach().numpy(), rtol=1e-10, atol=1e-10)
    dx, dw, db = J.norm_backward(dy, s, w, mean, rstd)
    (gx,) = torch.autograd.grad(ty, ts, torch.tensor(dy))
    assert np.allclose(dx, gx.numpy(), rtol=1e-8, atol=1e-8)
    for i in range(B):                                                     # each sample's own gradient
        ws, bs = tw.clone().requires_grad_(True), tb.clone().requires_grad_(True)
        ti = torch.nn.functional.layer_norm(torch.tensor(s[i]), (n,), ws, bs, eps=float(np.float32(1e-5)))
        gw, gb = torch.autograd.grad(ti, (ws, bs), torch.tensor(dy[i]))
        assert np.allclose(dw[i], gw.numpy(), rtol=1e-9, atol=1e-9) and np.allclose(db[i], gb.numpy(), rtol=1e-9)


def test_rms_norm_against_differences():
    B, T, n = 2, 3, 9
    x, dy, w = _rows(B, T, n, 5), _rows(B, T, n, 6), 1 + 0.1 * _rows(1, 1, n, 7)[0, 0]
    res, p, h = _rows(B, T, n, 8), 0.3, 1e-6

    def loss(x, res, w):
        s = J.dropout(x, SEED, SITE, p, res=res)
        return (J.norm(s, w, rms=True)[0] * dy).sum() + 0.5 * (s * s).sum()
    s = J.dropout(x, SEED, SITE, p, res=res)
    _, _, rstd = J.norm(s, w, rms=True)
    dx, dw, _ = J.norm_backward(dy, s, w, None, rstd, ds=s)
    dh = J.dropout(dx, SEED, SITE, p)
    rng = np.random.default_rng(9)
    for arr, grad, which in ((x, dh, 0), (res, dx, 1), (w, dw.sum(0), 2)):
        v = rng.standard_normal(arr.shape)
        args = [x, res, w]
        up, dn = list(args), list(args)
        up[which], dn[which] = arr + h * v, arr - h * v
        assert abs((loss(*up) - loss(*dn)) / (2 * h) - (grad * v).sum()) <= 1e-6 * max(1.0, abs((grad * v).sum()))


def test_vectors():
    G = np.array([[3.0, 4.0], [np.nan, np.inf], [1.0, -1.0]])
    assert np.array_equal(J.norm_vectors(G)[[0, 2]], [25.0, 2.0])
    assert np.array_equal(J.clip_accumulate_vectors(G, [0.5, 0.0, 2.0]), [3.5, 0.0])
