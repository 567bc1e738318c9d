"""The joint norm of many tensors and their clipping against the 64-bit oracle.

Tolerance, u = 2^-24 and r = 2^-8 for bf16 results (0 for fp32): the norm is exact to 64 bits but for its rounding, u;
the threshold (fp32 in the C interface), the factor and the product are rounded once each, (1 + u)^3 - 1 < 3.01 u, and r of
the result.
"""

import math

import numpy as np
import pytest
import torch

from oracle import head as O
from oracle.estimators import as_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
R = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}


@pytest.fixture(scope="module")
def D():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc
    dprc.lib()
    return dprc


def make(shapes, seed=0, dtypes=(torch.float32,), scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(s, generator=g)).to(dtypes[i % len(dtypes)]).cuda() for i, s in enumerate(shapes)]


def check(D, xs, max_norm, outs=None):
    ref, norm = O.clip([as_f64(x) for x in xs], max_norm)
    n1 = D.dprc_grad_norm(xs)
    got, n2 = D.dprc_grad_clip(xs, max_norm, outs=outs)
    assert torch.equal(n1, n2) and n1.shape == (1,)
    assert abs(n1.item() - norm) <= 1.01 * U * norm
    for y, x, z in zip(got, xs, ref):
        bad = ~(np.abs(as_f64(y) - z) <= (3.01 * U + R[x.dtype]) * np.abs(z) + 2.0 ** -149)
        assert not bad.any()


LISTS = [[(1,)], [(7,), (1, 1), (3, 5)], [(16384,), (16385,), (16383,)], [(111, 64), (64,), (64, 111), (1009, 64)],
         [(3, 5, 7), (2, 40001), (300, 300)], [(k + 1,) for k in range(47)], [(k % 9 + 1, 33) for k in range(48)],
         [(k % 9 + 1, 33) for k in range(49)], [(17, k + 1) for k in range(160)], [(1 << 20,), (5,), (1500, 1111)]]


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("shapes", LISTS)
def test_lists(D, shapes, dtypes):
    xs = make(shapes, seed=len(shapes), dtypes=dtypes)
    n = math.sqrt(sum(math.prod(s) for s in shapes))
    for max_norm in (0.3 * n, 10.0 * n + 1):
        check(D, xs, max_norm, [torch.empty_like(x) for x in xs])
    check(D, [x.clone() for x in xs], 0.5 * n, [torch.empty_like(x) for x in xs])
    ys = [x.clone() for x in xs]
    D.dprc_grad_clip(ys, 0.3 * n)                        # in place
    out, _ = D.dprc_grad_clip(xs, 0.3 * n, outs=[torch.empty_like(x) for x in xs])
    assert all(torch.equal(a, b) for a, b in zip(ys, out))
    keep = [x.clone() for x in xs]
    D.dprc_grad_clip(xs, 10.0 * n + 1)
    assert all(torch.equal(a, b) for a, b in zip(xs, keep))


def test_strided_rows(D):
    base = [torch.full((50, 133), 9.0, device="cuda"), torch.full((3, 40000), 9.0, device="cuda").bfloat16(),
            torch.full((30000, 3), 9.0, device="cuda")]
    xs = [base[0][:, :130], base[1][:, 1:20001], base[2][:, :2]]
    for x, y in zip(xs, make([x.shape for x in xs])):
        x.copy_(y)
    outs = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in xs]
    check(D, xs, 10.0, outs)
    want, _ = D.dprc_grad_clip([x.contiguous() for x in xs], 10.0)
    D.dprc_grad_clip(xs, 10.0)
    assert all(torch.equal(x, w) for x, w in zip(xs, want))
    assert (base[0][:, 130:] == 9).all() and (base[1][:, 20001:] == 9).all() and (base[1][:, 0] == 9).all()
    assert (base[2][:, 2:] == 9).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(2, 4), (3, 70), (5, 9000)])
def test_rows_as_far_apart_as_the_tensor_is_long(D, R, C, dtype):
    """A row stride of R C elements, on either side of a contiguous tensor: nothing between the rows is read or written."""
    n, x = R * C, make([(R, C)], seed=C, dtypes=(dtype,))[0]
    want, norm = D.dprc_grad_clip([x], 0.5, outs=[torch.empty_like(x)])
    buf = torch.full((R, n), 7.0, dtype=dtype, device="cuda")
    out, m = D.dprc_grad_clip([x], 0.5, outs=[buf[:, :C]])
    assert torch.equal(out[0], want[0]) and torch.equal(m, norm) and (buf[:, C:] == 7).all()
    buf = torch.full((R, n), float("nan"), dtype=dtype, device="cuda")
    buf[:, :C] = x
    out, m = D.dprc_grad_clip([buf[:, :C]], 0.5, outs=[torch.empty_like(x)])
    assert torch.equal(out[0], want[0]) and torch.equal(m, D.dprc_grad_norm([buf[:, :C]]))
    check(D, [buf[:, :C]], 0.5, [torch.empty_like(x)])


def test_odd_addresses(D):
    buf, out = torch.randn(5003, device="cuda").bfloat16(), torch.zeros(5003, device="cuda").bfloat16()
    check(D, [buf[1:], buf[:1]], 3.0, [out[1:], out[:1]])
    fl, fo = torch.randn(4097, device="cuda"), torch.zeros(4097, device="cuda")
    check(D, [fl[3:]], 3.0, [fo[1:4095]])


def test_extremes(D):
    """Squares that no fp32 value holds, zeros, values that are not finite, and empty tensors."""
    check(D, make([(1000,), (37,)], scale=1e30), 1.0, [torch.empty(1000, device="cuda"), torch.empty(37, device="cuda")])
    check(D, make([(1000,)], scale=1e-30), 1e-31, [torch.empty(1000, device="cuda")])
    z, n = D.dprc_grad_clip([torch.zeros(100, device="cuda")], 1.0)
    assert n.item() == 0 and not z[0].any()
    top = torch.full((1 << 16,), 3e38, device="cuda")                 # the norm is past fp32
    y, n = D.dprc_grad_clip([top], 2.56, outs=[torch.empty_like(top)])
    assert n.item() == math.inf
    np.testing.assert_allclose(as_f64(y[0]), 0.01, rtol=3 * U)
    for bad in (math.nan, math.inf, -math.inf):
        xs = make([(100,), (50, 50)], dtypes=(torch.bfloat16, torch.float32))
        xs[1][3, 4] = bad
        ys, n = D.dprc_grad_clip(xs, 1.0, outs=[torch.full_like(x, 5.0) for x in xs])
        assert not math.isfinite(n.item()) and not any(y.any() for y in ys)
        D.dprc_grad_clip(xs, 1.0)
        assert not any(x.any() for x in xs)
    xs = [torch.empty(0, device="cuda"), torch.ones(4, device="cuda"), torch.empty(3, 0, device="cuda")]
    check(D, xs, 1.0, [torch.empty_like(x) for x in xs])
    assert D.dprc_grad_norm([torch.empty(0, device="cuda")]).item() == 0
    assert D.dprc_grad_clip([torch.empty(0, device="cuda")], 1.0)[1].item() == 0


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)])
def test_several_launches_past_the_caches(D, dtypes):
    """More tensors than a launch takes and more than 300 MiB: every launch reads past the caches but for its end."""
    gen = torch.Generator(device="cuda").manual_seed(len(dtypes))
    shapes = [(1201, 1571 + 4 * k) if k % 7 else (3 * k + 1,) for k in range(110)]
    xs = [torch.randn(s, generator=gen, device="cuda").to(dtypes[i % len(dtypes)]) for i, s in enumerate(shapes)]
    assert sum(x.numel() * x.element_size() for x in xs) > 300 << 20
    norm = math.sqrt(sum(x.double().square().sum().item() for x in xs))
    want = D.dprc_grad_norm(xs)
    assert abs(want.item() - norm) <= 1.01 * U * norm
    for max_norm in (0.3 * norm, 10.0 * norm):
        c = min(1.0, max_norm / norm)
        outs, n = D.dprc_grad_clip(xs, max_norm, outs=[torch.full_like(x, 9.0) for x in xs])
        assert torch.equal(n, want)
        for x, y in zip(xs, outs):
            z = c * x.double()
            assert ((y.double() - z).abs() <= (3.01 * U + R[x.dtype]) * z.abs() + 2.0 ** -149).all()
    ys, _ = D.dprc_grad_clip([x.clone() for x in xs], 0.3 * norm)       # in place
    outs, _ = D.dprc_grad_clip(xs, 0.3 * norm, outs=[torch.empty_like(x) for x in xs])
    assert all(torch.equal(a, b) for a, b in zip(ys, outs))


def test_past_32_bits(D):
    """More than 2^31 elements in one tensor, and rows more than 2^31 elements apart."""
    big = torch.zeros(2 ** 31 + 20000, dtype=torch.bfloat16, device="cuda")
    big[-1], big[0], big[2 ** 31 + 5] = 3.0, 4.0, 12.0
    _, n = D.dprc_grad_clip([big], 6.5)
    assert n.item() == 13.0
    assert (big[-1], big[0], big[2 ** 31 + 5]) == (1.5, 2.0, 6.0)
    rows = big.as_strided((2, 8), (2 ** 31 + 19992, 1))
    assert D.dprc_grad_norm([rows]).item() == 2.5


def test_captured(D):
    xs = make([(1000, 33), (77,)], dtypes=(torch.float32, torch.bfloat16))
    src = [x.clone() for x in xs]
    outs = [torch.empty_like(x) for x in xs]
    D.dprc_grad_clip(xs, 5.0, outs=outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, n = D.dprc_grad_clip(xs, 5.0, outs=outs)
    for f in (1.0, 0.001, 3.0):
        for x, s in zip(xs, src):
            x.copy_(f * s)
        graph.replay()
        got = [y.clone() for y in outs] + [n.clone()]
        torch.cuda.synchronize()
        want, m = D.dprc_grad_clip(xs, 5.0, outs=[torch.empty_like(x) for x in xs])
        assert all(torch.equal(a, b) for a, b in zip(got, want + [m]))
