"""Layer norm forward and backward against the formula in 64 bits, element by element.

Bounds, with u = 2^-24: a sum of n values by a workgroup of 256 is a chain of at most n / 256 + 16 additions (or, by a
wavefront, n / 64 + 16), each off by at most u of what is summed so far, so it is off by at most (16 + n / 64) u times
the sum of magnitudes; differences of values carry the error of the mean, products a u each.  The rounding to bf16
(binary16) is off by at most half a unit in the last place of 8 (11)
significant bits, 2^-8 (2^-11) of the value, for binary16 at least 2^-25."""
import math

import numpy as np
import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import LayerNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
EPS = 1e-5


def rounded(ref, err, dtype):
    """bound of a value `err` off that is rounded to dtype"""
    return err + HALF_ULP[dtype] * (ref.abs() + err) + SMALLEST[dtype]


def within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / bound)[bad].max()):.3g} of the bound"


def make(rows, cols, dtype, w, pad=0, shift=0, mean=0.3, seed=1):
    """x, dy with rows cols + pad apart that begin `shift` values into their memory; weight, bias"""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def rows_of(scale, add):
        flat = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=dtype, device=DEV)
        view = flat[shift:].view(rows, cols + pad)[:, :cols]
        view.copy_(torch.empty(rows, cols, device=DEV).normal_(generator=gen) * scale + add)
        return view

    weight = (1 + 0.2 * torch.empty(cols, device=DEV).normal_(generator=gen)).to(w)
    bias = (0.2 * torch.empty(cols, device=DEV).normal_(generator=gen)).to(w)
    return rows_of(1.5, mean), rows_of(0.7, 0.0), weight, bias


def check_forward(x, weight, bias, y, mean, rstd):
    n = x.shape[1]
    X = x.double()
    w = torch.ones(n, device=DEV).double() if weight is None else weight.double()
    b = torch.zeros(n, device=DEV).double() if bias is None else bias.double()
    mu = X.mean(1, keepdim=True)
    var = (X - mu).square().mean(1, keepdim=True)
    rs = (var + EPS).rsqrt()
    chain = (16 + n / 64) * U
    e_mu = chain * X.abs().mean(1, keepdim=True)
    # (the variance is of differences that are e_mu + U |x| off, which shifts their mean square by the square of the shift)
    e_var = 2 * chain * var + (e_mu + U * X.abs().amax(1, keepdim=True)).square() + 4 * U * var.sqrt() * X.abs().amax(1, keepdim=True)
    e_rs = rs * (e_var / (2 * (var + EPS)) + 4 * U)
    xh = (X - mu) * rs
    e_xh = (e_mu + U * (X - mu).abs()) * rs + (X - mu).abs() * e_rs + 2 * U * xh.abs()
    ref = xh * w + b
    within(y, ref, rounded(ref, e_xh * w.abs() + 2 * U * ((xh * w).abs() + b.abs()), y.dtype), "y")
    if mean is not None:
        within(mean, mu[:, 0], e_mu[:, 0] + 1e-40, "mean")
        within(rstd, rs[:, 0], e_rs[:, 0], "rstd")


def check_backward(dy, x, weight, mean, rstd, dx, dweight, dbias):
    """(for the mean and rstd that the forward pass gave)"""
    rows, n = x.shape
    D = dy.double()
    w = torch.ones(n, device=DEV).double() if weight is None else weight.double()
    mu, rs = mean.double()[:, None], rstd.double()[:, None]
    xh = (x.double() - mu) * rs
    a = D * w
    e_xh = 3 * U * xh.abs()
    chain = (18 + n / 64) * U
    m1, m2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    e1, e2 = chain * a.abs().mean(1, keepdim=True), (chain + 3 * U) * (a * xh).abs().mean(1, keepdim=True)
    if dx is not None:
        ref = rs * (a - m1 - xh * m2)
        err = rs * (e1 + e2 * xh.abs() + e_xh * m2.abs() + 6 * U * (a.abs() + m1.abs() + (xh * m2).abs()))
        within(dx, ref, rounded(ref, err, dx.dtype), "dx")
    # (a column's sum is a chain of at most one addition for every row and 32 more)
    column = (32 + rows) * U
    if dweight is not None:
        ref = (D * xh).sum(0)
        within(dweight, ref, rounded(ref, (column + 4 * U) * (D * xh).abs().sum(0), dweight.dtype), "dweight")
    if dbias is not None:
        ref = D.sum(0)
        within(dbias, ref, rounded(ref, column * D.abs().sum(0), dbias.dtype), "dbias")


def run(rows, cols, dtype, w, pad=0, shift=0, mean=0.3):
    x, dy, weight, bias = make(rows, cols, dtype, w, pad, shift, mean)
    whole = torch.full((rows, cols + pad), -7.0, dtype=dtype, device=DEV)
    y = whole[:, :cols]
    mu, rs = (torch.full((rows,), float("nan"), device=DEV) for _ in range(2))
    cs.cs_layer_norm(x, weight, bias, y, mu, rs, EPS)
    check_forward(x, weight, bias, y, mu, rs)
    assert (whole[:, cols:] == -7.0).all()
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    whole = torch.full((rows, cols + pad), -7.0, dtype=dtype, device=DEV)
    dx, dw, db = whole[:, :cols], torch.full_like(weight, float("nan")), torch.full_like(bias, float("nan"))
    cs.cs_layer_norm_grad(dy, x, weight, mu, rs, dx, dw, db, ws)
    check_backward(dy, x, weight, mu, rs, dx, dw, db)
    assert (whole[:, cols:] == -7.0).all()


SHAPES = [(1, 1), (3, 1), (1, 2), (5, 3), (2, 4), (4, 5), (7, 7), (3, 8), (2, 9), (65, 16), (130, 63), (1, 64), (33, 100), (2, 511),
          (1, 512), (700, 512), (5, 513), (19, 1000), (9, 1024), (3, 1025), (300, 2047), (17, 2048), (4, 2049), (2, 4096),
          (6, 5000), (3, 8192), (2, 8200), (3, 16384), (2, 20001), (1, 40000)]


@pytest.mark.parametrize("dtype,w", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_backward(rows, cols, dtype, w):
    run(rows, cols, TYPES[dtype], TYPES[w])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (3, 5), (7, 3), (8, 0), (16, 8)])
@pytest.mark.parametrize("cols", [6, 64, 333, 1024, 2500, 9001])
def test_strides_and_alignments(cols, pad, shift, dtype):
    run(11, cols, TYPES[dtype], torch.float32, pad, shift)


@pytest.mark.parametrize("rows,cols", [(4097, 64), (20_001, 8), (9000, 192), (3000, 1030), (66_000, 3)])
def test_many_rows(rows, cols):
    run(rows, cols, torch.bfloat16, torch.float32)


def test_a_mean_much_larger_than_the_spread():
    run(9, 777, torch.float32, torch.float32, mean=1000.0)
    run(9, 33_000, torch.float32, torch.float32, mean=1000.0)


def test_without_weights_statistics_and_single_gradients():
    x, dy, weight, bias = make(37, 600, torch.float32, torch.float32)
    y = torch.empty_like(x)
    cs.cs_layer_norm(x, None, None, y, None, None, EPS)
    check_forward(x, None, None, y, None, None)
    cs.cs_layer_norm(x, weight, None, y, None, None, EPS)
    check_forward(x, weight, None, y, None, None)
    mu, rs = (torch.empty(37, device=DEV) for _ in range(2))
    cs.cs_layer_norm(x, None, bias, y, mu, rs, EPS)
    check_forward(x, None, bias, y, mu, rs)
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(37, 600), dtype=torch.uint8, device=DEV)
    for keep in ("dx", "dweight", "dbias"):
        out = {"dx": torch.empty_like(x), "dweight": torch.empty_like(weight), "dbias": torch.empty_like(bias)}
        out = {k: v if k == keep else None for k, v in out.items()}
        cs.cs_layer_norm_grad(dy, x, None, mu, rs, out["dx"], out["dweight"], out["dbias"], None if keep == "dx" else ws)
        check_backward(dy, x, None, mu, rs, **out)


@pytest.mark.parametrize("cols", [5, 256, 3000, 17_000])
def test_in_place_gives_the_same_bits(cols):
    x, dy, weight, bias = make(23, cols, torch.bfloat16, torch.float32, pad=2)
    y, mu, rs = torch.empty(23, cols, dtype=x.dtype, device=DEV), *(torch.empty(23, device=DEV) for _ in range(2))
    cs.cs_layer_norm(x, weight, bias, y, mu, rs, EPS)
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(23, cols), dtype=torch.uint8, device=DEV)
    dx, dw, db = torch.empty_like(y), torch.empty_like(weight), torch.empty_like(bias)
    cs.cs_layer_norm_grad(dy, x, weight, mu, rs, dx, dw, db, ws)

    def copy(t):
        whole = torch.zeros(23, cols + 2, dtype=t.dtype, device=DEV)
        whole[:, :cols] = t
        return whole[:, :cols]

    own = copy(x)
    cs.cs_layer_norm(own, weight, bias, own, None, None, EPS)
    assert torch.equal(own, y)
    for into_dy in (True, False):
        d, xx, dw2, db2 = copy(dy), copy(x), torch.empty_like(dw), torch.empty_like(db)
        cs.cs_layer_norm_grad(d, xx, weight, mu, rs, d if into_dy else xx, dw2, db2, ws)
        assert torch.equal(d if into_dy else xx, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_the_same_call_gives_the_same_bits():
    x, dy, weight, bias = make(5003, 515, torch.bfloat16, torch.float32)
    ln = LayerNorm(weight, bias, 5003, x.dtype, EPS)
    got = []
    for _ in range(3):
        y = ln.forward(x).clone()
        got.append((y, ln.backward(dy).clone(), ln.dweight.clone(), ln.dbias.clone()))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_no_rows():
    w = torch.ones(40, device=DEV)
    x = torch.empty(0, 40, device=DEV)
    cs.cs_layer_norm(x, w, w, torch.empty_like(x), None, None, EPS)
    dw, db = torch.full_like(w, 3.0), torch.full_like(w, 3.0)
    none = torch.empty(0, device=DEV)
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(0, 40), dtype=torch.uint8, device=DEV)
    cs.cs_layer_norm_grad(x, x, w, none, none, torch.empty_like(x), dw, db, ws)
    assert not dw.any() and not db.any()


def test_values_that_are_not_finite_stay_in_their_row():
    x, dy, weight, bias = make(6, 900, torch.float32, torch.float32)
    x[1, 5], x[3, 800] = math.nan, math.inf
    y, mu, rs = torch.empty_like(x), *(torch.empty(6, device=DEV) for _ in range(2))
    cs.cs_layer_norm(x, weight, bias, y, mu, rs, EPS)
    assert y[1].isnan().all() and y[3].isnan().all()
    keep = [0, 2, 4, 5]
    check_forward(x[keep], weight, bias, y[keep], mu[keep], rs[keep])
    dx = torch.empty_like(x)
    cs.cs_layer_norm_grad(dy, x, weight, mu, rs, dx, None, None, None)
    check_backward(dy[keep], x[keep], weight, mu[keep], rs[keep], dx[keep], None, None)


def test_gradient_against_differences():
    """loss = sum y q, in steps of h along random directions: (f(x + h v) - f(x - h v)) / 2h is h^2 |f'''| / 6 and the rounding
    of two sums of y, about 2^-24 sqrt(n) |q| each, over 2h, off the gradient's product with v"""
    x, q, weight, bias = make(8, 64, torch.float32, torch.float32)
    ln = LayerNorm(weight, bias, 8)
    ln.forward(x)
    dx, dw, db = ln.backward(q.contiguous()).clone(), ln.dweight.clone(), ln.dbias.clone()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    h = 2.0 ** -6

    def f(xx, w, b):
        y = torch.empty_like(xx)
        cs.cs_layer_norm(xx, w, b, y, None, None, EPS)
        return float((y.double() * q.double()).sum())

    for name, grad in (("x", dx), ("weight", dw), ("bias", db)):
        at = {"x": x.contiguous(), "weight": weight, "bias": bias}
        v = torch.empty_like(grad).normal_(generator=gen)
        up, down = dict(at), dict(at)
        up[name], down[name] = at[name] + h * v, at[name] - h * v
        slope = (f(up["x"], up["weight"], up["bias"]) - f(down["x"], down["weight"], down["bias"])) / (2 * h)
        want = float((grad.double() * v.double()).sum())
        scale = float((grad.double() * v.double()).abs().sum())
        assert abs(slope - want) <= 5e-3 * scale, (name, slope, want, scale)


def test_on_another_stream():
    x, dy, weight, bias = make(400, 384, torch.float32, torch.float32)
    ln = LayerNorm(weight, bias, 400)
    want = [ln.forward(x).clone(), ln.backward(dy.contiguous()).clone(), ln.dweight.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [ln.forward(x).clone(), ln.backward(dy.contiguous()).clone(), ln.dweight.clone()]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals():
    x = torch.zeros(4, 16, device=DEV)
    y, w = torch.zeros_like(x), torch.ones(16, device=DEV)
    mu = torch.zeros(4, device=DEV)
    for bad in (dict(x=x.double()), dict(x=x[:, ::2], y=y[:, ::2], w=w[:8]), dict(w=w[:8]), dict(w=w.half()), dict(y=y.bfloat16()),
                dict(mean=mu), dict(mean=mu[:3], rstd=mu[:3]), dict(x=x.cpu()), dict(y=x[:, :16].flatten().as_strided((4, 16), (16, 1), 0)[[0, 1, 2]])):
        a = dict(x=x, y=y, w=w, mean=None, rstd=None) | bad
        with pytest.raises(cs.CsError):
            cs.cs_layer_norm(a["x"], a["w"], None, a["y"], a["mean"], a["rstd"], EPS)
    wide = torch.zeros(4, 40, device=DEV)
    cs.cs_layer_norm(wide[:, :16], w, w, wide[:, 16:32], None, None, EPS)       # two slices of the same rows lie apart
    with pytest.raises(cs.CsError):
        cs.cs_layer_norm(wide[:, :16], w, w, wide[:, 8:24], None, None, EPS)
    with pytest.raises(cs.CsError):
        cs.cs_layer_norm_grad(x, x, w, mu, mu, y, w.clone(), w.clone(), torch.empty(8, dtype=torch.uint8, device=DEV))
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(4, 16), dtype=torch.uint8, device=DEV)
    with pytest.raises(cs.CsError):
        cs.cs_layer_norm_grad(x, x, w, mu, mu, y, w, w.clone(), ws)             # the gradient over the weight itself
    with pytest.raises(cs.CsError):
        LayerNorm(w, w, 4).backward(x)
