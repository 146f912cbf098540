"""The policy loss of a batch of no tokens: sums are 0, and nothing of the batch before is left."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import PolicyLoss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE = torch.empty(0)


def nan(*shape):
    return torch.full(shape, math.nan, device=DEV)


def workspaces():
    return [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (0, 64)]


def test_policy_loss_of_no_tokens():
    e = NONE.to(DEV)
    for ws in workspaces():
        sums = nan(4)
        cs.cs_policy_loss(cs.CsPolicy(0.25, 0.25, 0.5, 0.5), e, e, e, e, e, e, e, e, e, sums, ws)
        assert sums.tolist() == [0.0] * 4
        cs.cs_policy_loss(cs.CsPolicy(0.25, 0.25, 0.0, 0.0), e, None, e, None, e, e, None, None, None, None, ws)      # (no sums are wanted)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_policy_loss_from_no_logits(dtype):
    e, target = NONE.to(DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    x = torch.empty(0, 1000, dtype=dtype, device=DEV)
    for ws in workspaces():
        sums = nan(4)
        cs.cs_token_policy_loss(cs.CsPolicy(0.25, 0.25, 0.5, 0.5), x, target, e, e, e, e, e, e, e, e, sums, torch.empty_like(x), ws)
        assert sums.tolist() == [0.0] * 4
        cs.cs_token_policy_loss(cs.CsPolicy(0.25, 0.25, 0.0, 0.0), x, target, e, None, e, e, e, e, e, None, None, x, ws)


def test_policy_object_after_a_batch():
    loss = PolicyLoss(8, 100, kl=0.5)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(8, 100, device=DEV, generator=gen)
    t = torch.arange(8, device=DEV)
    old, ref, a, w = (torch.randn(8, device=DEV, generator=gen) - 5 for _ in range(4))
    assert loss.loss(x, t, old, ref, a, w)[0].any()
    sums, dx = loss.loss(x[:0], t[:0], old[:0], ref[:0], a[:0], w[:0])
    assert sums.tolist() == [0.0] * 4 and dx.shape == (0, 100)
    assert loss.of_logprobs(old, None, old, ref, a, w)[0].any()
    sums, g, h = loss.of_logprobs(old[:0], None, old[:0], ref[:0], a[:0], w[:0])
    assert sums.tolist() == [0.0] * 4 and len(g) == len(h) == 0
    empty = PolicyLoss(0, 100)
    assert empty.loss(x[:0], t[:0], old[:0], None, a[:0], w[:0])[0].tolist() == [0.0] * 4


def test_policy_loss_of_no_tokens_in_a_graph():
    e, ws, sums = NONE.to(DEV), torch.empty(64, dtype=torch.uint8, device=DEV), nan(4)

    def call():
        cs.cs_policy_loss(cs.CsPolicy(0.25, 0.25, 0.0, 0.0), e, None, e, None, e, e, None, None, None, sums, ws)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        sums.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        assert sums.tolist() == [0.0] * 4
