"""Lists of matrices that share memory: parts of one array may stand side by side, but nothing that is written may be another matrix's."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import Muon, Orthogonalizer
from test_gpu_muon import matrices_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_side_by_side():
    """columns of one array, every other matrix of a stack, rows"""
    x = matrices_of(6, 70, 90)
    want = []
    for part in (x[0, :, :40], x[0, :, 40:], x[1::2], x[2::2], x[0, :0]):
        want.append(torch.empty(part.shape, device=DEV))
        Orthogonalizer([part], [want[-1]]).run()
    both = torch.full_like(x, math.nan)
    places = [both[0, :, :40], both[0, :, 40:], both[1::2], both[2::2], both[0, :0]]
    Orthogonalizer([x[0, :, :40], x[0, :, 40:], x[1::2], x[2::2], x[0, :0]], places).run()
    for a, b in zip(places, want):
        assert (a - b).abs().max().item() <= 1e-5 if a.numel() else True
    assert torch.isfinite(both).all()


def test_one_in_the_other():
    x, y = matrices_of(2, 70, 90), torch.empty(2, 70, 90, device=DEV)
    for outputs in ([y[0], y[0, 1:, :]], [y, y[1]], [y[0, :, :50], y[0, :, 49:]], [y.view(-1)[:6300].view(70, 90), y.view(-1)[6200:12500].view(70, 90)]):
        with pytest.raises(cs.CsError, match="overlap"):
            Orthogonalizer([torch.zeros_like(o) for o in outputs], outputs)
    with pytest.raises(cs.CsError, match="overlap"):
        Orthogonalizer([x[0], x[1]], [x[1], x[0]])       # (one would be written before it is read)
    Orthogonalizer([x[0], x[1]], [x[0], x[1]])
    m = torch.zeros(3, 70, 90, device=DEV)
    with pytest.raises(cs.CsError, match="overlap"):
        Muon([y[0], y[1]], [x[0], x[1]], m=[m[0], m.view(-1)[6299:12599].view(70, 90)])
    with pytest.raises(cs.CsError, match="overlap"):
        Muon([y[0], y[1]], [x[0], y[0]], m=[m[0], m[1]])
    opt = Muon([y[0], y[1]], [x[0], x[1]], m=[m[0], m[1]])
    with pytest.raises(cs.CsError, match="overlap"):
        opt.set_grads([x[0], m[0]])
    opt.step()                                           # (the list is the one that it was)
