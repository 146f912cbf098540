"""The backward pass over its own inputs (dx is x, or dy) where a workgroup has several rows and the last one has not enough: the groups
without a row left have nothing to do with a row that another group is writing.  Its gradient overflows here, and must not reach the
weights' gradients: they are the same bits as with dx apart."""
import pytest
import torch

import paper_1903_04488_amd as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("over", ["x", "dy"])
@pytest.mark.parametrize("rows", [1025, 1501, 9003])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("cols", [100, 500, 1000, 1999])
def test_rows_that_a_group_does_not_have(cols, dtype, rows, over):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.empty(rows, cols, device=DEV).normal_(generator=gen).to(dtype) for _ in range(2))
    mean, rstd = x.float().mean(1), 1 / x.float().std(1)
    big = 6e4 if dtype == torch.float16 else 3e38
    dy[-1, ::2], dy[-1, 1::2] = big, -big
    rstd[-1] = 50.0 if dtype == torch.float16 else 2.0
    weight = torch.ones(cols, device=DEV)
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    def run(dx, x, dy):
        dw, db = torch.empty_like(weight), torch.empty_like(weight)
        cs.cs_layer_norm_grad(dy, x, weight, mean, rstd, dx, dw, db, ws)
        return dx, dw, db

    want = run(torch.empty_like(x), x, dy)
    assert int((~torch.isfinite(want[0][-1])).sum()) > cols // 2 and torch.isfinite(want[0][:-1]).all()
    assert torch.isfinite(want[1]).all() or dtype == torch.bfloat16
    for _ in range(3):
        a, b = x.clone(), dy.clone()
        got = run(a if over == "x" else b, a, b)
        assert all(torch.equal(p.nan_to_num(nan=7.0), q.nan_to_num(nan=7.0)) for p, q in zip(got, want))
