"""The binding's checks of given outputs (no GPU): what would have the library read or write past a
tensor's end is refused before anything is enqueued."""

import types

import pytest
import torch

from paper_2605_24879_amd import dprc


@pytest.fixture
def calls(monkeypatch):
    """A library that records its calls, for host tensors in the place of device ones."""
    seen = []

    def entry(name):
        if name.endswith("_workspace"):
            return lambda *a: 0
        return lambda *a: seen.append((name, a)) or dprc.SUCCESS
    monkeypatch.setattr(dprc, "lib", lambda: types.SimpleNamespace(**{n: entry(n) for n in dprc.EXPORTS}))
    monkeypatch.setattr(dprc, "_stream", lambda dev: None)
    return seen


def test_per_sample_gradients_need_a_row_each(calls):
    x, st = torch.zeros(4, 3, 8), torch.zeros(12)
    back = lambda **kw: dprc.dprc_layernorm_backward(x, x, None, st, st, **kw)
    one = torch.zeros(1, 8)
    overlapping = torch.zeros(64).as_strided((4, 8), (7, 1))
    for bad in (one.expand(4, 8), overlapping):
        for kw in (dict(dw=bad), dict(db=bad), dict(dw=bad, db=bad), dict(dw=bad, db=torch.zeros(4, 8))):
            with pytest.raises(ValueError):
                back(**kw)
    assert not calls
    # rows of a buffer, and one sample's row at any stride
    G = torch.zeros(4, 20)
    back(dw=G[:, :8], db=G[:, 9:17])
    assert calls[-1][0] == "dprc_layernorm_backward" and calls[-1][1][15] == 20
    x, st = x[:1], st[:3]
    for dw in (one, one.expand(1, 8), G[1:2, 3:11], torch.zeros(64).as_strided((1, 8), (0, 1))):
        dprc.dprc_layernorm_backward(x, x, None, st, st, dw=dw)
        assert calls[-1][1][15] == 8


@pytest.fixture
def layers(monkeypatch):
    """Two layers' (A, E) of four samples as the binding sees them, host tensors for device ones."""
    monkeypatch.setattr(dprc, "make_layer", lambda A, E, layer_id: dprc.Layer())
    return [(torch.zeros(4, 2, 6), torch.zeros(4, 2, 5), j) for j in range(2)]


def test_per_sample_values_need_an_entry_each(calls, layers):
    full, A, E = torch.zeros(4), layers[0][0], layers[0][1]
    uses = {
        "n2": [lambda v: dprc.dprc_norm_hutch(layers, 4, 0, n2=v), lambda v: dprc.dprc_norm_hutch(layers, 4, 0, n2=v, accumulate=True),
               lambda v: dprc.dprc_norm_hutch_clip(layers, 4, 0, 1.0, n2=v, accumulate=True),
               lambda v: dprc.dprc_norm_hutch_clip_static(layers, 4, 0, 1.0, n2=v),
               lambda v: dprc.dprc_norm_hutchpp(layers, 4, 4, 0, n2=v, accumulate=True)],
        "c": [lambda v: dprc.dprc_norm_hutch_clip(layers, 4, 0, 1.0, c=v), lambda v: dprc.dprc_norm_hutch_clip_static(layers, 4, 0, 1.0, c=v),
              lambda v: dprc.dprc_clip_scale(full, 1.0, c=v), lambda v: dprc.dprc_clip_accumulate(A, E, v),
              lambda v: dprc.dprc_clip_accumulate_layers(layers, v)],
    }
    for name, fs in uses.items():
        for k, f in enumerate(fs):
            for bad in (torch.zeros(1), torch.zeros(3), torch.zeros(1).expand(4), torch.zeros(8)[::2], full.double(), full.bfloat16(),
                        torch.zeros(4, device="meta")):
                with pytest.raises(ValueError):
                    f(bad)
                    pytest.fail(f"{name} use {k} was taken")
    for f in (lambda v: dprc.dprc_norm_hutch(layers, 4, 0, n2_layers=v), lambda v: dprc.dprc_norm_hutch_clip(layers, 4, 0, 1.0, n2_layers=v),
              lambda v: dprc.dprc_norm_hutch_clip_static(layers, 4, 0, 1.0, n2_layers=v),
              lambda v: dprc.dprc_norm_hutchpp(layers, 4, 4, 0, n2_layers=v)):
        for bad in (torch.zeros(7), torch.zeros(4, 2).t(), torch.zeros(2, 4).double()):
            with pytest.raises(ValueError):
                f(bad)
    for bad in (torch.zeros(8)[::2], full.double()):                  # the estimates that clip factors are made from
        with pytest.raises(ValueError):
            dprc.dprc_clip_scale(bad, 1.0)
    assert not calls
    for ok in (full, torch.zeros(9), torch.zeros(9)[2:6], torch.zeros(2, 2)):
        for f in uses["n2"] + uses["c"]:
            f(ok)
    assert len(calls) == 40
    dprc.dprc_norm_hutch(layers, 4, 0, n2_layers=torch.zeros(2, 4))
    assert calls[-1][0] == "dprc_norm_hutch"


def test_the_sum_outlives_a_norm_in_the_inputs_place(calls):
    # without a residual and dropout s is x, unless y is written over x: then s is a tensor of its own
    x, v = torch.randn(2, 3, 8), torch.ones(8)
    was = x.clone()
    _, s, _, _ = dprc.dprc_layernorm(x, v)
    assert s is x and calls[-1][1][5] is None
    for y in (x, x.view(2, 3, 8)):
        got, s, _, _ = dprc.dprc_layernorm(x, v, y=y)
        a = calls[-1][1]
        assert got is y and s.data_ptr() != x.data_ptr() and a[5] == s.data_ptr() and a[7] == x.data_ptr()
    given = torch.empty_like(x)
    assert dprc.dprc_layernorm(x, v, y=x, s=given)[1] is given
    assert torch.equal(x, was)


def test_a_workspace_has_to_hold_its_bytes(monkeypatch):
    # many entries over few bytes are no workspace
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    fine = torch.zeros(64)
    assert dprc._workspace(256, None, fine) is fine and dprc._workspace(256, None, torch.zeros(2, 40)).numel() == 80
    for bad in (torch.zeros(1).expand(64), torch.zeros(1, 16).expand(4, 16), torch.zeros(128)[::2], torch.zeros(63)):
        with pytest.raises(ValueError):
            dprc._workspace(256, None, bad)
