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
