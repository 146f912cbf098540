"""The loss's gradient in rows whose logits lie far from 0: what probabilities are made of is differences of logits, so nothing in
the bounds (tests/far_logits.py) grows with the logits themselves."""
import pytest
import torch

import paper_1903_04488_amd as cs
from far_logits import DEV, TYPES, far_rows, wanted, within

pytestmark = pytest.mark.gpu


def loss(x, target, g, h, scale, out=None):
    rows = len(x)
    dx = torch.full_like(x, -7.0) if out is None else out
    ws = torch.empty(cs.cs_token_workspace_bytes(rows, x.shape[1], 0), dtype=torch.uint8, device=DEV)
    cs.cs_token_loss(x, target, g, h, *(torch.empty(rows, device=DEV) for _ in range(3)), dx, ws, scale)
    return dx


def coefficients(rows):
    gen = torch.Generator(device=DEV).manual_seed(7)
    return torch.empty(rows, device=DEV).normal_(generator=gen), torch.empty(rows, device=DEV).normal_(generator=gen)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(24, 40), (13, 1000), (30, 5000), (600, 5001), (12, 30_001)])
def test_rows_held_by_a_wavefront_or_a_workgroup(rows, vocab, dtype):
    x, target = far_rows(rows, vocab, TYPES[dtype])
    for scale, entropy_too in ((1.0, True), (0.7, True), (1.3, False)):
        g, h = coefficients(rows)
        h = h if entropy_too else None
        ref, bound = wanted(x, target, g, h, scale, False)
        dx = loss(x, target, g, h, scale)
        within(dx, ref, bound, "loss")
        same = x.clone()
        assert torch.equal(loss(same, target, g, h, scale, same), dx)


@pytest.mark.parametrize("dtype,vocab", [("f32", 66_001), ("bf16", 131_500)])
def test_rows_that_no_workgroup_holds(dtype, vocab):
    x, target = far_rows(1030, vocab, TYPES[dtype])
    g, h = coefficients(1030)
    dx = loss(x, target, g, h, 0.9)
    for at in range(0, 1030, 103):
        some = slice(at, at + 103)
        ref, bound = wanted(x[some], target[some], g[some], h[some], 0.9, False)
        within(dx[some], ref, bound, "loss")
