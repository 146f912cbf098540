"""A layer norm without a bias: the results of a bias of zeros, by the short way through the binding's checks."""
import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd import binding
from paper_1903_04488_amd.training import LayerNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_the_short_way_and_the_same_bits(monkeypatch):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy, weight = (torch.randn(s, device=DEV, generator=gen) for s in ((40, 96), (40, 96), (96,)))
    with_bias, without = LayerNorm(weight, torch.zeros(96, device=DEV), 40), LayerNorm(weight, None, 40)
    y, dx = with_bias.forward(x).clone(), with_bias.backward(dy).clone()

    def long_way(*_):
        raise AssertionError("the long way")

    monkeypatch.setattr(binding, "_rows", long_way)
    assert torch.equal(without.forward(x), y) and torch.equal(without.backward(dy), dx)
    assert torch.equal(without.dweight, with_bias.dweight) and without.dbias is None


@pytest.mark.parametrize("bad", [7, "cpu", "double", "short", "apart"])
def test_a_bias_that_is_wrong_is_refused(bad):
    x, w = torch.zeros(4, 96, device=DEV), torch.ones(96, device=DEV)
    bias = {"cpu": w.cpu(), "double": w.double(), "short": w[:95], "apart": torch.ones(192, device=DEV)[::2]}.get(bad, bad)
    with pytest.raises(cs.CsError):
        cs.cs_layer_norm(x, w, bias, torch.empty_like(x))
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(4, 96), dtype=torch.uint8, device=DEV)
    mean = torch.zeros(4, device=DEV)
    with pytest.raises(cs.CsError):
        cs.cs_layer_norm_grad(x, x, w, mean, mean + 1, torch.empty_like(x), torch.empty_like(w), bias, ws)
