"""Rows that the policy loss from logits leaves out (weight 0, or no target): their logits may hold anything, and their gradient is 0, so
that nothing of them reaches the weights."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from test_gpu_policy_loss import HIGH, LOW, TYPES, fused, tokens_of
from test_gpu_token_logprobs import logits_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows of a wavefront, of 256, 512 and 1024 threads, few that are not held, rows in parts, a stream
SIZES = [(9, 64), (9, 1000), (600, 3000), (300, 9001), (40, 20_000), (9, 40_003), (9, 70_001), (6, 140_000), (1025, 140_001), (1030, 70_001)]


@pytest.mark.parametrize("rows,vocab,dtype", [(*s, t) for s in SIZES for t in TYPES if s[0] * s[1] < 1 << 26 or (t == "bf16") == (s[1] > 1e5)])
@pytest.mark.parametrize("kl,bonus", [(0.0, 0.0), (0.0625, 0.03125)])
def test_what_rows_left_out_hold(rows, vocab, dtype, kl, bonus):
    x, target = logits_of(rows, vocab, TYPES[dtype], seed=rows + vocab)
    x = x.contiguous()
    t = tokens_of(rows, seed=3)
    target.clamp_(0, vocab - 1)
    base = fused(x, target, t, 0.0, 0.0, 0.75)[0]
    t["old"], t["ref"] = (base + t[k] - t["logp"] for k in ("old", "ref"))
    t["w"] = t["w"] + 0.125
    out = [0, 1, 2, 3, rows - 1]
    target[1] = -1
    target[3] = vocab
    t["w"][[0, 2, rows - 1]] = 0.0
    logp, entropy, lse, loss, sums, dx = fused(x, target, t, kl, bonus, 0.75)
    assert (dx[out] == 0).all() and torch.isfinite(dx.float()).all()
    bad = x.clone()
    bad[0, vocab // 2] = math.nan
    bad[1] = math.nan
    bad[2, -1] = math.inf
    bad[3] = math.inf
    bad[rows - 1] = -math.inf
    for in_place in (False, True):
        *_, got_loss, got_sums, got = fused(bad.clone(), target, t, kl, bonus, 0.75, in_place=in_place)
        assert torch.equal(got, dx) and torch.equal(got_loss, loss) and torch.equal(got_sums, sums)
    # a row that counts is not spared
    bad[4, 5] = math.nan
    assert torch.isnan(fused(bad, target, t, kl, bonus, 0.75)[-1][4]).all()
