"""The preference loss of no pairs: sums are 0, no token has a gradient, and nothing of the batch before is left."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import PreferenceLoss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE = torch.empty(0)


def nan(*shape):
    return torch.full(shape, math.nan, device=DEV)


def workspaces():
    return [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (0, 64)]


@pytest.mark.parametrize("tokens", [0, 1, 1023, 5000, 3_000_001])
def test_preference_loss_of_no_pairs(tokens):
    logp, e = torch.zeros(tokens, device=DEV), NONE.to(DEV)
    begin = torch.zeros(1, dtype=torch.int64, device=DEV)
    for ws in workspaces():
        sums, whole = nan(3), torch.full((tokens + 2,), 7.0, device=DEV)
        g = whole[1:1 + tokens]
        cs.cs_preference_loss(cs.CsPreference(0, 0, 0.5, 0.0, 0.0), logp, None, None, begin, None, e, e, g, sums, ws)
        assert sums.tolist() == [0.0] * 3 and (g == 0).all() and whole[0] == whole[-1] == 7.0
        sums = nan(3)
        cs.cs_preference_loss(cs.CsPreference(0, 0, 0.5, 0.0, 0.0), logp, None, None, begin, None, e, e, None, sums, ws)
        assert sums.tolist() == [0.0] * 3


def test_preference_object_after_a_batch():
    loss = PreferenceLoss(100, 4, beta=0.5)
    logp = -torch.rand(100, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    sums, g = loss.loss(logp, None, torch.tensor([0, 20, 30, 70, 100], device=DEV))
    assert sums.any() and g.all()
    sums, g = loss.loss(logp[:60], None, torch.zeros(1, dtype=torch.int64, device=DEV))
    assert sums.tolist() == [0.0] * 3 and len(g) == 60 and (g == 0).all()
    sums, g = PreferenceLoss(100, 0).loss(logp, None, torch.zeros(1, dtype=torch.int64, device=DEV))
    assert sums.tolist() == [0.0] * 3 and (g == 0).all()


def test_no_pairs_refuse_what_pairs_refuse():
    logp, e = torch.zeros(100, device=DEV), NONE.to(DEV)
    begin, ws = torch.zeros(1, dtype=torch.int64, device=DEV), torch.empty(64, dtype=torch.uint8, device=DEV)
    both = torch.zeros(100, device=DEV)
    for g, sums in ((logp, nan(3)), (both, both[10:13])):
        with pytest.raises(cs.CsError):
            cs.cs_preference_loss(cs.CsPreference(0, 0, 0.5, 0.0, 0.0), logp, None, None, begin, None, e, e, g, sums, ws)
