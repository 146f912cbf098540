"""Scales near the end of binary32, whose product with log2(e) is no number any more: the differences that they multiply are 0
or decide everything."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [50, 3000, 70_000])
def test_a_scale_near_the_end_of_binary32(vocab):
    x = torch.zeros(4, vocab, device=DEV)
    x[1, 7] = 1.0
    x[2] = 1.0
    x[3] = -1.0
    target = torch.full((4,), 7, dtype=torch.int64, device=DEV)
    logp, entropy, lse = (torch.empty(4, device=DEV) for _ in range(3))
    ws = torch.empty(cs.cs_token_workspace_bytes(4, vocab, 0), dtype=torch.uint8, device=DEV)
    cs.cs_token_logprobs(x, target, logp, entropy, lse, None, None, ws, 3e38)
    want = torch.full((4,), -math.log(vocab), device=DEV)
    want[1] = 0.0
    torch.testing.assert_close(logp, want, rtol=1e-5, atol=1e-6)
    torch.testing.assert_close(entropy, -want, rtol=1e-5, atol=1e-6)
    g = torch.full((4,), 1e-38, device=DEV)
    later, both = torch.empty_like(x), torch.empty_like(x)
    cs.cs_token_logprobs_grad(x, target, lse, None, g, None, later, 3e38)
    cs.cs_token_loss(x, target, g, None, logp, entropy, lse, both, ws, 3e38)
    for dx in (later, both):
        assert torch.isfinite(dx).all() and not dx[1].any()
        for row in (0, 2, 3):
            torch.testing.assert_close(dx[row, :7], torch.full((7,), -3.0 / vocab, device=DEV), rtol=1e-4, atol=0)
