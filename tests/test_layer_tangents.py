"""Forward-mode derivatives are refused by the layers, as those of backward mode are (no GPU: the refusal comes before any of
the layer's work)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2608_13255_amd import multiview

NAMES = {multiview.MultiViewAttention: ("w_qkv", "w_out", "q_gain", "k_gain"),
         multiview.MultiViewBlock: ("w_qkv", "w_out", "w_in", "w_down", "b_in", "q_gain", "k_gain", "attention_gain", "feed_gain")}


class Reached(Exception):
    """The layer went on to its work."""


def layer_of(kind, monkeypatch):
    layer = object.__new__(kind)
    layer.B, layer.N, layer.H, layer.W, layer.width, layer.dtype = 1, 2, 3, 4, 8, torch.float32
    layer.foreground = torch.ones((1, 2, 3, 4), dtype=torch.bool)
    for name in ("b_qkv", "b_out", "b_in", "b_down"):
        setattr(layer, name, None)
    for name in NAMES[kind]:
        setattr(layer, name, torch.ones(8))

    def slice(self, views):
        raise Reached
    monkeypatch.setattr(kind, "slice", slice)
    return layer


CASES = [(kind, name) for kind in NAMES for name in ("x",) + NAMES[kind]]


@pytest.mark.parametrize("kind,name", CASES)
def test_tangents_are_refused(monkeypatch, kind, name):
    layer = layer_of(kind, monkeypatch)
    x = torch.randn((1, 1, 3, 4, 8))
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
        if name != "x":
            setattr(layer, name, dual(getattr(layer, name)))
        got = dual(x) if name == "x" else x
        assert not got.requires_grad
        for grad in (True, False):      # (no_grad() stops only backward mode)
            with torch.set_grad_enabled(grad), pytest.raises(ValueError, match="no gradient"):
                layer(got, [1])
        with torch.inference_mode(), pytest.raises(Reached):
            layer(got, [1])


@pytest.mark.parametrize("kind", NAMES)
def test_without_tangents_it_goes_on(monkeypatch, kind):
    layer = layer_of(kind, monkeypatch)
    x = torch.randn((1, 1, 3, 4, 8))
    with pytest.raises(Reached):
        layer(x, [1])
    with forward_ad.dual_level(), pytest.raises(Reached):
        layer(x, [1])


@pytest.mark.parametrize("kind", NAMES)
def test_jvp_is_refused(monkeypatch, kind):
    layer = layer_of(kind, monkeypatch)
    x = torch.randn((1, 1, 3, 4, 8))
    with pytest.raises(ValueError, match="no gradient"):
        torch.func.jvp(lambda t: layer(t, [1]), (x,), (torch.ones_like(x),))
    with pytest.raises(ValueError, match="no gradient"):
        torch.func.grad(lambda t: layer(t, [1]).sum())(x)
