"""Log probability and entropy of rows whose logits lie far from 0: both are made of differences of logits, so their bounds do not
grow with the logits.

Bounds, u = 2^-24, d = z - max z, E = sum p |d|: a sum of exponentials is off by L = u (20 + n / 256 + 4 E), the target's d by 4 u of
itself; the entropy is ln of that sum and E, a quotient of two such sums."""
import numpy as np
import pytest
import torch

import paper_1903_04488_amd as cs
from far_logits import DEV, TYPES, U, far_rows, within

pytestmark = pytest.mark.gpu


def check(x, target, scale):
    rows, vocab = x.shape
    logp, entropy, lse = (torch.empty(rows, device=DEV) for _ in range(3))
    ws = torch.empty(cs.cs_token_workspace_bytes(rows, vocab, 0), dtype=torch.uint8, device=DEV)
    cs.cs_token_logprobs(x, target, logp, entropy, lse, None, None, ws, scale)
    z = x.double() * float(np.float32(scale))
    d = z - z.amax(1, keepdim=True)
    e = d.exp()
    log_sum = e.sum(1, keepdim=True).log()
    E = torch.where(e > 0, e * d.abs(), 0.0).sum(1, keepdim=True) / e.sum(1, keepdim=True)
    L = U * (20 + vocab / 256 + 4 * E)
    at = d.gather(1, target[:, None])
    fits = at[:, 0] > -3e38                              # (a difference beyond binary32 is -inf)
    within(logp[fits][:, None], (at - log_sum)[fits], (L + 4 * U * (at.abs() + log_sum))[fits], "logp")
    within(entropy[:, None], log_sum + E, 2 * L * (1 + E) + 4 * U * (log_sum + E), "entropy")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(24, 40), (13, 1000), (30, 5000), (1100, 5001), (12, 70_001), (12, 300_007)])
def test_rows_far_from_0(rows, vocab, dtype):
    x, target = far_rows(rows, vocab, TYPES[dtype])
    for scale in (1.0, 0.7, 1.3):
        check(x, target, scale)


def test_many_long_rows_far_from_0():
    """by a workgroup of 256 each: sums of 258 terms a thread, relative to a number that may be 100 from the largest product"""
    x, target = far_rows(1030, 66_001, torch.float32)
    for scale in (0.9, 1.0):
        check(x, target, scale)
