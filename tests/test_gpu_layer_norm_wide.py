"""Gradients of weight and bias of rows that have more columns than one launch has threads for (2^26 for the sums of the shares, 2^30, the
most there are, for the shares themselves).  Of one row they are products and copies: dw = dy xh, off by 4 u and the rounding to binary16."""
import pytest
import torch

import paper_1903_04488_amd as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("cols", [(1 << 26) - 3, (1 << 26) + 5, 1 << 30])
def test_gradients_of_weight_and_bias_of_very_wide_rows(cols):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.empty(1, cols, dtype=torch.float16, device=DEV).normal_(generator=gen) for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device=DEV), torch.full((1,), 0.75, device=DEV)
    dw, db = (torch.full((cols,), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(1, cols), dtype=torch.uint8, device=DEV)
    cs.cs_layer_norm_grad(dy, x, None, mean, rstd, None, dw, db, ws)
    assert torch.equal(db, dy[0])
    for at in range(0, cols, 1 << 26):
        part = slice(at, at + (1 << 26))
        want = dy[0, part].double() * ((x[0, part].double() - 0.25) * 0.75)
        off = (dw[part].double() - want).abs()
        assert (off <= want.abs() * (4 * U + 2.0 ** -11) + 2.0 ** -25).all()
