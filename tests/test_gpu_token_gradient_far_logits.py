"""The gradient that is asked for after the forward pass, and the loss of rows that several workgroups share (which takes that way), in
rows whose logits lie far from 0: an lse in binary32 says little or nothing there.  Bounds: tests/far_logits.py."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from far_logits import DEV, TYPES, far_rows, wanted, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(24, 40), (13, 1000), (30, 5000), (600, 5001), (12, 70_001), (12, 300_007)])
def test_gradients_asked_for_later(rows, vocab, dtype):
    x, target = far_rows(rows, vocab, TYPES[dtype])
    gen = torch.Generator(device=DEV).manual_seed(7)
    g, h = (torch.empty(rows, device=DEV).normal_(generator=gen) for _ in range(2))
    logp, entropy, lse = (torch.empty(rows, device=DEV) for _ in range(3))
    ws = torch.empty(cs.cs_token_workspace_bytes(rows, vocab, 0), dtype=torch.uint8, device=DEV)
    for scale, h in ((1.0, h), (0.7, h), (1.3, None)):
        ref, bound = wanted(x, target, g, h, scale, True)
        cs.cs_token_logprobs(x, target, logp, entropy, lse, None, None, ws, scale)
        dx = torch.full_like(x, -7.0)
        cs.cs_token_logprobs_grad(x, target, lse, None if h is None else entropy, g, h, dx, scale)
        within(dx, ref, bound, "gradient")
        same = x.clone()                                 # over the logits themselves
        cs.cs_token_logprobs_grad(same, target, lse, None if h is None else entropy, g, h, same, scale)
        assert torch.equal(same, dx)
        if ws.numel():
            cs.cs_token_loss(x, target, g, h, logp, entropy, lse, dx, ws, scale)
            within(dx, ref, bound, "loss")
            same = x.clone()
            cs.cs_token_loss(same, target, g, h, logp, entropy, lse, same, ws, scale)
            assert torch.equal(same, dx)


def test_a_row_of_the_lowest_value_is_not_an_empty_one():
    """its products with the scale leave binary32: its lse is the lowest number, and -inf stays the mark of rows with no token"""
    x = torch.full((3, 900), torch.finfo(torch.float32).min, device=DEV)
    x[1] = -math.inf
    x[2] = 0.5
    target = torch.zeros(3, dtype=torch.int64, device=DEV)
    logp, entropy, lse = (torch.empty(3, device=DEV) for _ in range(3))
    cs.cs_token_logprobs(x, target, logp, entropy, lse, None, None, torch.empty(0, dtype=torch.uint8, device=DEV), 2.0)
    assert lse[0] == torch.finfo(torch.float32).min and lse[1] == -math.inf and logp[1] == -math.inf and entropy[1] == 0
    assert float(logp[0]) == pytest.approx(-math.log(900), rel=1e-6) and float(entropy[0]) == pytest.approx(math.log(900), rel=1e-6)
    one, dx = torch.ones(3, device=DEV), torch.empty_like(x)
    cs.cs_token_logprobs_grad(x, target, lse, None, one, None, dx, 2.0)
    assert not dx[1].any()
    for row in (0, 2):
        assert float(dx[row, 0]) == pytest.approx(2 - 2 / 900, rel=1e-5)
        torch.testing.assert_close(dx[row, 1:], torch.full((899,), -2 / 900, device=DEV), rtol=1e-5, atol=0)
