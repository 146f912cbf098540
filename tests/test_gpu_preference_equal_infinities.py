"""A token that neither the model nor its reference allows, in the loss of pairs, in one launch and by pieces.  Beta is 1/2, and every token that counts is -1 with a reference of -1/2, or without one."""
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


@pytest.mark.parametrize("pairs", [3, 40])
@pytest.mark.parametrize("kind", ["logistic", "hinge", "square"])
@pytest.mark.parametrize("mean", [False, True])
def test_a_token_that_neither_model_allows(pairs, kind, mean):
    """equal infinities are 0 apart, as they are in the policy loss: the token counts with a ratio of 1"""
    t = batch(pairs, True)
    for side in (0, 3 * pairs):
        same = t | {"logp": t["logp"].clone(), "ref": t["ref"].clone()}
        same["logp"][side + 4] = same["ref"][side + 4] = -0.5
        want = run(same, kind, BETA, mean=mean)
        for v in (-INF, INF):
            same["logp"][side + 4] = same["ref"][side + 4] = v
            got = run(same, kind, BETA, mean=mean)
            for k in want:
                assert torch.isfinite(want[k]).all() and torch.equal(got[k], want[k]), k
