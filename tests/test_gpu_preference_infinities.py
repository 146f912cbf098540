"""Log probabilities of -inf (a token that a mask rules out) in the loss of pairs: what the formula gives in the limit, in one launch and by
pieces.  Beta is 1/2, and every token that counts is -1 with a reference of -1/2, or without one."""
import math

import pytest
import torch

from test_gpu_preference_loss import run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = math.inf
BETA = 0.5


def batch(pairs, reference):
    """pairs of answers of 3 and 2 tokens: rewards -3/4 and -1/2 with the reference, -3/2 and -1 without"""
    begin = torch.tensor([0] + [3] * pairs + [2] * pairs, device=DEV).cumsum(0)
    logp = torch.full((5 * pairs,), -1.0, device=DEV)
    return {"logp": logp, "ref": torch.full_like(logp, -0.5) if reference else None, "counts": None, "begin": begin, "w": None}


def loss_of(z, kind, smoothing):
    """(loss, slope) at an infinite z"""
    if kind == "logistic":
        def soft(v):
            return max(v, 0.0)
        terms = [f * soft(v) for f, v in ((1 - smoothing, -z), (smoothing, z)) if f]
        return sum(terms), smoothing - (0.0 if z > 0 else 1.0)
    if kind == "hinge":
        return (0.0, 0.0) if z > 0 else (INF, -1.0)
    return INF, z


# (few pairs are one launch, more go by pieces)
@pytest.mark.parametrize("pairs", [3, 40])
@pytest.mark.parametrize("reference", [False, True])
@pytest.mark.parametrize("kind,smoothing", [("logistic", 0.0), ("logistic", 1.0), ("logistic", 0.25), ("hinge", 0.0), ("square", 0.0)])
@pytest.mark.parametrize("rejected", [False, True])
def test_a_token_that_cannot_be(pairs, reference, kind, smoothing, rejected):
    t = batch(pairs, reference)
    plain = run(t, kind, BETA, smoothing)
    at = 3 * pairs + 2 if rejected else 4                # in answers of pair 1
    t["logp"][at] = -INF
    got = run(t, kind, BETA, smoothing)
    loss, slope = loss_of(INF if rejected else -INF, kind, smoothing)
    assert got["loss"][1] == loss and got["reward"][1 + (pairs if rejected else 0)] == -INF
    assert got["sums"][0] == (INF if loss == INF else got["loss"].double().sum().float())
    assert got["sums"][2] == (INF if rejected else -INF)
    assert (got["g_logp"][3:6] == BETA * slope).all() and (got["g_logp"][3 * pairs + 2:3 * pairs + 4] == -BETA * slope).all()
    # the others are as they were
    others = torch.arange(pairs, device=DEV) != 1
    assert torch.equal(got["loss"][others], plain["loss"][others])
    tokens = torch.ones(5 * pairs, dtype=torch.bool, device=DEV)
    tokens[3:6] = tokens[3 * pairs + 2:3 * pairs + 4] = False
    assert torch.equal(got["g_logp"][tokens], plain["g_logp"][tokens])


@pytest.mark.parametrize("pairs", [3, 40])
def test_what_has_no_limit_is_not_a_number(pairs):
    """both answers of a pair cannot be; infinities of both signs"""
    t = batch(pairs, False)
    t["logp"][[3, 3 * pairs + 2]] = -INF
    got = run(t, "logistic", BETA)
    assert torch.isnan(got["loss"][1]) and torch.isnan(got["sums"][0]) and torch.isnan(got["g_logp"][3:6]).all() and torch.isfinite(got["g_logp"][:3]).all()
    t = batch(pairs, False)
    t["logp"][3], t["logp"][4] = -INF, INF
    got = run(t, "hinge", BETA)
    assert torch.isnan(got["reward"][1]) and torch.isnan(got["loss"][1]) and torch.isfinite(got["loss"][2:]).all()
