"""Dropout and norms past 32-bit counts of pieces and of elements, and the launches of the junction
operators as the launch trace records them."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import junction as J
from oracle.estimators import as_f64

pytestmark = pytest.mark.gpu

SEED, SITE = 0x1122334455667788, 6


@pytest.fixture(scope="module")
def D():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24879_amd import dprc
    dprc.lib()
    return dprc


def _free(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of free memory")


def test_dropout_of_two_to_the_31_pieces(D):
    # 2^28 + 3 rows of 64 bf16: 2^31 + 24 pieces, more workgroups than a grid's first row holds
    _free(40)
    R, n, p = (1 << 28) + 3, 64, 0.25
    x = torch.ones(1, R, n, dtype=torch.bfloat16, device="cuda")
    D.dprc_dropout(x, p, SEED, SITE, out=x)
    for r0 in (0, 12345678, (1 << 27) - 2, (1 << 28) - 4, R - 5):
        ref = J.dropout_factors(SEED, SITE, 5, n, p, row0=r0)
        assert np.array_equal(as_f64(x[0, r0:r0 + 5]), as_f64(torch.from_numpy(ref).bfloat16())), r0
    # dropped with probability 1/4: 2^34 elements, five standard deviations
    kept = sum(int((x[0, k:k + (1 << 24)] != 0).sum()) for k in range(0, R, 1 << 24))
    assert abs(kept / (R * n) - 0.75) <= 5 * np.sqrt(0.25 * 0.75 / (R * n))


def test_norm_of_rows_past_32_bit_elements(D):
    # 2^27 + 5 rows of 40: more than 2^32 elements
    _free(60)
    R, n = (1 << 27) + 5, 40
    g = torch.Generator().manual_seed(1)
    base = torch.randn(64, n, generator=g).bfloat16().cuda()
    x = base.repeat((R + 63) // 64, 1)[:R].view(1, R, n)
    w = (1 + 0.1 * torch.randn(n, generator=g)).cuda()
    y, s, mean, rstd = D.dprc_layernorm(x, w)
    small = D.dprc_layernorm(base.view(1, 64, n), w)
    for r0 in (0, 64 * 1000003, R - R % 64 - 64):
        assert torch.equal(y[0, r0:r0 + 64], small[0][0]) and torch.equal(mean[r0:r0 + 64], small[2])
    assert torch.equal(y[0, R - 5:], small[0][0, :5])
    del y
    dx, _, dw, db = D.dprc_layernorm_backward(x, s, w, mean, rstd)
    ref = D.dprc_layernorm_backward(base.view(1, 64, n), small[1], w, small[2], small[3])
    for r0 in (0, 64 * 1000003, R - R % 64 - 64):
        assert torch.equal(dx[0, r0:r0 + 64], ref[0][0])
    # sums of R terms: every token's chain is at most R / 256 rounds long in any of the parts
    _, m64, r64 = J.norm(base.view(1, 64, n))
    _, one_w, one_b = J.norm_backward(base.view(1, 64, n), base.view(1, 64, n), w, mean[:64], rstd[:64])
    tail_w, tail_b = J.norm_backward(base[:5].view(1, 5, n), base[:5].view(1, 5, n), w, mean[:5], rstd[:5])[1:]
    full = R // 64
    for got, one, tail, mag in ((dw, one_w, tail_w, (np.abs(as_f64(base)) * 4).sum(0)), (db, one_b, tail_b, np.abs(as_f64(base)).sum(0))):
        want = full * one + tail
        assert np.all(np.abs(as_f64(got) - want) <= (R / 256) * 2.0 ** -24 * full * mag)


def _trace(D, fn, capacity=16):
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2 * capacity)]
    for e in events:
        e.record()                                     # torch creates an event when it is first recorded
    torch.cuda.synchronize()
    ptrs = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    kinds, count = (ctypes.c_int32 * capacity)(), ctypes.c_int32(0)
    D.dprc_trace_launches(ctypes.cast(ptrs, ctypes.c_void_p), ctypes.cast(kinds, ctypes.c_void_p), capacity,
                          ctypes.cast(ctypes.byref(count), ctypes.c_void_p))
    try:
        fn()
    finally:
        n = count.value
        D.dprc_trace_launches(None, None, 0, None)
    torch.cuda.synchronize()
    return [D.KERNEL_NAMES[k] for k in kinds[:n]], [events[2 * j].elapsed_time(events[2 * j + 1]) for j in range(n)]


def _back(D, B, T, n):
    x = torch.randn(B, T, n, device="cuda")
    _, s, mean, rstd = D.dprc_layernorm(x)
    return lambda: D.dprc_layernorm_backward(x, s, None, mean, rstd)


CALLS = {
    "dropout": (lambda D: lambda: D.dprc_dropout(torch.ones(1, 9, 70, device="cuda"), 0.1, 1, 2), ["dropout"]),
    "norm": (lambda D: lambda: D.dprc_layernorm(torch.ones(1, 9, 70, device="cuda")), ["layernorm"]),
    "norm, long rows": (lambda D: lambda: D.dprc_layernorm(torch.ones(1, 2, 20001, device="cuda")), ["layernorm"]),
    "backward, whole samples": (lambda D: _back(D, 3, 9, 300), ["layernorm_backward"]),
    "backward, cut samples": (lambda D: _back(D, 3, 900, 300), ["layernorm_backward"] * 2),
    "backward, a workgroup's rows": (lambda D: _back(D, 2, 5, 9000), ["layernorm_backward"]),
    "backward, a workgroup's rows, cut samples": (lambda D: _back(D, 2, 50, 9000), ["layernorm_backward"] * 2),
    "backward, long rows": (lambda D: _back(D, 2, 5, 20000), ["layernorm_backward"] * 2),
    "backward, long rows, cut samples": (lambda D: _back(D, 2, 50, 20000), ["layernorm_backward"] * 3),
    "vector norms": (lambda D: lambda: D.dprc_norm_vectors(torch.ones(4, 300, device="cuda")), ["vector_norms"]),
    "vector norms, split": (lambda D: lambda: D.dprc_norm_vectors(torch.ones(4, 300000, device="cuda")), ["vector_norms"] * 2),
    "vector sums": (lambda D: lambda: D.dprc_clip_accumulate_vectors(torch.ones(4, 300, device="cuda"), torch.ones(4, device="cuda")),
                    ["vector_sums"]),
    "vector sums, split": (lambda D: lambda: D.dprc_clip_accumulate_vectors(torch.ones(5000, 30, device="cuda"),
                                                                            torch.ones(5000, device="cuda")), ["vector_sums"] * 2),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_every_launch_is_recorded(D, name):
    make, kinds = CALLS[name]
    got, ms = _trace(D, make(D))
    assert got == kinds and all(t > 0 for t in ms)


@pytest.mark.parametrize("dtype,n", [("bf16", 512), ("bf16", 1024), ("bf16", 2048), ("bf16", 4096), ("bf16", 8192), ("f32", 512),
                                     ("f32", 1024), ("f32", 2048), ("f32", 4096), ("f32", 8192), ("bf16", 16384)])
def test_calls_that_stream_past_the_caches_give_the_same_bits(D, dtype, n):
    # tensors of 320 MiB together take non-temporal accesses; rows of the same call in pieces do not
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    R = (320 << 20) // (2 * n * (2 if dtype == "bf16" else 4)) + 3
    g = torch.Generator(device="cuda").manual_seed(n)
    x, z = (torch.randn(1, R, n, generator=g, device="cuda").to(dt) for _ in range(2))
    w = (1 + 0.1 * torch.randn(n, generator=g, device="cuda")).to(dt)
    cut = [(0, 100), (R // 2, R // 2 + 57), (R - 33, R)]
    for kw in (dict(res=z, p=0.0), dict(p=0.0), dict(res=z, p=0.1, seed=SEED, site_id=SITE), dict(p=0.1, seed=SEED, site_id=SITE)):
        y, s, mean, rstd = D.dprc_layernorm(x, w, **kw)
        for a, b in cut:
            # the mask goes by the row: the piece starts at row 0, so it is compared where there is none
            if kw["p"] == 0.0:
                part = dict(kw, res=z[:, a:b]) if "res" in kw else kw
                for u, v in zip((y[:, a:b], s[:, a:b], mean[a:b], rstd[a:b]), D.dprc_layernorm(x[:, a:b], w, **part)):
                    assert torch.equal(u, v)
        if kw["p"] > 0.0:
            for u, v in zip((y[:, :100], s[:, :100]), D.dprc_layernorm(x[:, :100], w, **dict(kw, **({"res": z[:, :100]} if "res" in kw else {})))):
                assert torch.equal(u, v)
            f = torch.from_numpy(J.dropout_factors(SEED, SITE, 33, n, 0.1, row0=R - 33)).cuda()
            tail = f.float() * x[0, R - 33:].float() + (z[0, R - 33:].float() if "res" in kw else 0.0)
            assert torch.allclose(s[0, R - 33:].float(), tail, rtol=2.0 ** -8, atol=1e-6)
    for res in (z, None):
        out = D.dprc_dropout(x, 0.1, SEED, SITE, res=res)
        assert torch.equal(out[:, :100], D.dprc_dropout(x[:, :100], 0.1, SEED, SITE, res=None if res is None else res[:, :100]))
        assert torch.equal(out, D.dprc_layernorm(x, w, res=res, p=0.1, seed=SEED, site_id=SITE)[1])
