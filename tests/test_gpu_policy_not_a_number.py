"""A log probability that is not a number shows in the policy loss also where the token has no advantage."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("where", ["logp", "old"])
@pytest.mark.parametrize("kl", [0.0, 0.5])
def test_without_an_advantage(where, kl):
    """S = min(r A, clip(r) A) of a ratio that is not a number; of one beyond binary32 it is 0"""
    t = {k: torch.zeros(3, device=DEV) for k in ("logp", "old", "ref", "a")}
    t[where][1] = math.nan
    t["old"][2] = -200.0
    w = torch.ones(3, device=DEV)
    loss, g, sums = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV), torch.zeros(4, device=DEV)
    cs.cs_policy_loss(cs.CsPolicy(0.25, 0.25, kl, 0.0), t["logp"], None, t["old"], t["ref"], t["a"], w, loss, g, None, sums,
                      torch.empty(64, dtype=torch.uint8, device=DEV))
    assert torch.isnan(loss[1]) and torch.isnan(g[1]) and torch.isnan(sums[0])
    assert loss[[0, 2]].tolist() == [0.0, 0.0] and g[[0, 2]].tolist() == [0.0, 0.0]
