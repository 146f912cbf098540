"""Matrices orthogonalised by Newton-Schulz products, and the optimizer that does this with its momentum, against the same steps in 64
bits.

Bounds.  Roundings of the products' factors by half a step u of their type (binary16: 2^-11; two of them: 2^-22) are taken as independent, so that
an element of L R^T is off by a sum of independent errors, u sqrt(sum_k 2 l_ik^2 r_jk^2) in the mean square at most, and the whole product in
the 2-norm by u sqrt(2 sum_k |l_k|^2 |r_k|^2) with the columns' norms; sums in binary32 add 2^-24 sqrt(K) of the product and of that root.  A step's
error is raised by later steps by no more than the largest slope of their polynomials between 0 and the largest singular value
(a matrix function's derivative has the polynomial's divided differences as its values).  The bound is the sum of these, computed along the steps
in 64 bits, four times for what is not independent.  Results are rounded to their type once more.  A single element, of N, is off by 64 / sqrt(N) of
the whole at most (the errors of different elements are alike in size)."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import NEWTON_SCHULZ, Muon, Orthogonalizer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def steps_of(u, terms, coefs=NEWTON_SCHULZ, eps=1e-7):
    """(the result in 64 bits, the bound of its 2-norm error) of one matrix"""
    u = u.double().cpu()
    if not u.any():
        return u, 0.0
    tall = u.shape[0] > u.shape[1]
    x = (u.t() if tall else u) / (torch.linalg.matrix_norm(u) + eps)
    near, sums = 2.0 ** (-11 * terms), 2.0 ** -24

    def product(l, r):
        """l r^T and its bound"""
        root = (2 * (l.square().sum(0) * r.square().sum(0)).sum()).sqrt()
        return l @ r.t(), float(near * root + sums * math.sqrt(l.shape[1]) * (root + torch.linalg.matrix_norm(l @ r.t())))

    off = 2.0 ** -21 * float(torch.linalg.matrix_norm(x))
    for a, b, c in coefs:
        s = float(torch.linalg.matrix_norm(x, 2))
        A, e_a = product(x, x)
        A0 = A - torch.diag(A.diagonal())
        AA, e_aa = product(A0, A0)
        e_a += near * float(torch.linalg.matrix_norm(A0)) + sums * float(torch.linalg.matrix_norm(A))
        B = b * A + c * A @ A
        B0 = B - torch.diag(B.diagonal())
        e_b = (abs(b) + 2 * abs(c) * s * s) * e_a + abs(c) * e_aa + near * float(torch.linalg.matrix_norm(B0)) + 8 * sums * float(torch.linalg.matrix_norm(B))
        _, e_x = product(B0, x.t().contiguous())
        new = a * x + B @ x
        at = torch.linspace(0, s, 1001, dtype=torch.float64)
        slope = float((a + 3 * b * at ** 2 + 5 * c * at ** 4).abs().max())
        off = slope * off + s * e_b + e_x + 2.0 ** -21 * float(torch.linalg.matrix_norm(new))
        x = new
    return (x.t() if tall else x), 4 * off


def close(got, want, off, what="", rounded=True):
    """rounded: to got's type"""
    t = got.dtype
    got, want = got.double().cpu(), want.double().cpu()
    assert torch.isfinite(got).all(), what
    half = HALF_ULP[t] * want.abs() + SMALLEST[t] if rounded else torch.zeros_like(want)
    d = (got - want).abs()
    n = want.numel()
    assert float((d - half).clamp(min=0).square().sum().sqrt()) <= off * (1 + HALF_ULP[t]), (what, float((d - half).clamp(min=0).norm()), off)
    assert (d <= half + off * min(1.0, 64 / math.sqrt(n)) * (1 + HALF_ULP[t])).all(), what


def matrices_of(count, rows, cols, dtype=torch.float32, seed=1, steep=False):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(count, rows, cols, device=DEV, generator=gen)
    if steep:                                            # a few directions are much larger than the rest
        r = max(1, min(rows, cols) // 8)
        x += torch.randn(count, rows, r, device=DEV, generator=gen) @ torch.randn(count, r, cols, device=DEV, generator=gen) * 3
    return x.to(dtype)


# a workgroup's own (up to 64 x 256), in slabs, and in tiles of every size
SIZES = [(1, 1, 1), (1, 1, 70), (2, 70, 1), (1, 3, 5), (1, 64, 64), (2, 65, 63), (3, 30, 64), (2, 64, 128), (2, 127, 50), (1, 65, 65), (1, 64, 129), (1, 16, 300), (3, 130, 257), (2, 257, 128), (1, 200, 1000),
         (1, 512, 512),
         (1, 60, 4000), (3, 250, 50), (2, 256, 64), (20, 64, 4097), (7, 5000, 33), (2, 250, 3000), (1, 2100, 330), (5, 65, 5000)]


@pytest.mark.parametrize("count,rows,cols", SIZES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("terms", [1, 2])
def test_orthogonalized_matches_the_steps(count, rows, cols, dtype, terms):
    x = matrices_of(count, rows, cols, TYPES[dtype], seed=rows + cols, steep=True)
    out = torch.full_like(x, float("nan"))
    Orthogonalizer([x], [out], terms=terms).run()
    for i in range(count):
        want, off = steps_of(x[i], terms)
        close(out[i], want, off, (i, rows, cols))


@pytest.mark.parametrize("terms", [1, 2])
def test_many_matrices_of_many_shapes(terms):
    """shapes in any order, an empty stack among them"""
    check_shapes([(20, 300, 520), (1, 5, 7), (0, 4, 4), (3, 0, 6), (6, 640, 257), (2, 1, 1000)], terms)


@pytest.mark.parametrize("terms", [1, 2])
def test_as_many_matrices_as_larger_tiles_are_taken_for(terms):
    check_shapes([(60, 300, 520), (1, 5, 7), (2, 1100, 900), (1, 130, 1)], terms)


@pytest.mark.parametrize("terms", [1, 2])
def test_small_ones_thin_ones_and_others_in_one_list(terms):
    check_shapes([(6, 30, 1000), (4, 200, 300), (5, 64, 200), (1, 3000, 64), (4, 50, 20), (1, 65, 9000)], terms)


@pytest.mark.parametrize("terms", [1, 2])
def test_the_largest_tiles(terms):
    """as many that tiles of 256 fill the GPU"""
    check_shapes([(4, 2000, 2030), (30, 8, 60)], terms, every=9)


def check_shapes(shapes, terms, every=None):
    xs = [matrices_of(*s, seed=i) for i, s in enumerate(shapes)]
    outs = [torch.full_like(x, float("nan")) for x in xs]
    o = Orthogonalizer(xs, outs, terms=terms)
    o.run()
    for x, out in zip(xs, outs):
        for i in range(0, len(x), every or (13 if len(x) > 20 else 5)):
            if x[i].numel():
                want, off = steps_of(x[i], terms)
                close(out[i], want, off, tuple(x.shape))
    # alone, in other tiles (whose sums of squares are taken in another order: the norm's last bit may differ)
    one = torch.empty_like(xs[0][3])
    Orthogonalizer([xs[0][3]], [one], terms=terms).run()
    off = steps_of(xs[0][3], terms)[1]
    close(one, outs[0][3], 2 * off)


def test_singular_values_and_vectors():
    """what it is for: singular values from 0.02 of the norm on end between 0.6 and 1.3, singular vectors stay"""
    gen = torch.Generator().manual_seed(1)
    u = torch.linalg.qr(torch.randn(96, 96, generator=gen, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(200, 96, generator=gen, dtype=torch.float64))[0]
    s = torch.logspace(0, -1.2, 96, dtype=torch.float64)
    x = (u * s @ v.t()).float().to(DEV)
    out = torch.empty_like(x)
    Orthogonalizer([x], [out]).run()
    d = u.t() @ out.double().cpu() @ v
    assert 0.6 < float(d.diagonal().min()) and float(d.diagonal().max()) < 1.3
    assert float((d - torch.diag(d.diagonal())).abs().max()) < 1e-4


def test_other_coefficients_step_by_step():
    """the classic cubic step, which converges to the nearest orthogonal matrix, sixteen times; and one single step"""
    x = matrices_of(1, 40, 90, steep=False)
    for coefs in (((1.5, -0.5, 0.0),) * 16, ((3.4445, -4.7750, 2.0315),), ((2.0, -1.5, 0.5), (1.875, -1.25, 0.375))):
        for terms in (1, 2):
            out = torch.empty_like(x)
            Orthogonalizer([x], [out], coefs=coefs, terms=terms).run()
            want, off = steps_of(x[0], terms, coefs)
            close(out[0], want, off, (coefs[0], terms))


@pytest.mark.parametrize("count,rows,cols", [(1, 3, 300000), (2, 64, 8192), (1, 64, 8193), (1, 20000, 100), (9, 64, 8000)])
@pytest.mark.parametrize("terms", [1, 2])
def test_long_matrices(count, rows, cols, terms):
    """as many slabs as there may be of one matrix and in all, and more (which are tiles)"""
    x = matrices_of(count, rows, cols, steep=True)
    out = torch.full_like(x, float("nan"))
    Orthogonalizer([x], [out], terms=terms).run()
    for i in range(0, count, 4):
        want, off = steps_of(x[i], terms)
        close(out[i], want, off)


# in tiles, a workgroup's own, in slabs of columns
KINDS = [(70, 130), (40, 100), (50, 700)]


@pytest.mark.parametrize("rows,cols", KINDS)
@pytest.mark.parametrize("power", [-120, -60, 60, 100])
def test_sizes_of_the_numbers_do_not_matter(power, rows, cols):
    """scaled by a power of 2 the result has the same bits (eps 0)"""
    x = matrices_of(1, rows, cols)
    x = torch.where(x.abs() < 2.0 ** -6, 0.0, x)         # (no subnormal numbers)
    outs = []
    for f in (1.0, 2.0 ** power):
        outs.append(torch.empty_like(x))
        Orthogonalizer([x * f], [outs[-1]], eps=0.0).run()
    assert torch.equal(*outs)


@pytest.mark.parametrize("rows,cols", KINDS)
def test_zeros_and_what_is_not_finite_stay_in_their_matrix(rows, cols):
    x = matrices_of(5, rows, cols)
    clean = torch.empty_like(x)
    Orthogonalizer([x], [clean]).run()
    x[1] = 0.0
    x[2, 3, 4] = float("nan")
    x[3, -1, -1] = float("inf")
    out = torch.empty_like(x)
    Orthogonalizer([x], [out]).run()
    assert torch.equal(out[0], clean[0]) and torch.equal(out[4], clean[4])
    assert (out[1] == 0).all() and torch.isnan(out[2]).all() and torch.isnan(out[3]).all()
    x[1] = 0.0
    Orthogonalizer([x], [out], eps=0.0).run()
    assert (out[1] == 0).all()
    # rows and columns of zeros
    y = matrices_of(1, rows, cols)
    y[0, 5:-10] = 0.0
    y[0, :, cols * 3 // 4:] = 0.0
    got = torch.empty_like(y)
    Orthogonalizer([y], [got]).run()
    want, off = steps_of(y[0], 2)
    close(got[0], want, off)
    assert (got[0, 5:-10] == 0).all() and (got[0, :, cols * 3 // 4:] == 0).all()


@pytest.mark.parametrize("rows,cols", KINDS + [(130, 70), (100, 40), (700, 50)])
def test_strides_and_in_place(rows, cols):
    wide = torch.full((3, rows + 10, cols + 70), float("nan"), device=DEV)
    x = matrices_of(3, rows, cols)
    inside = wide[:, 4:4 + rows, 33:33 + cols]
    inside.copy_(x)
    want = torch.empty_like(x)
    Orthogonalizer([x], [want]).run()
    target = torch.full((3, rows + 20, cols + 10), 7.0, device=DEV)
    at = target[:, 10:10 + rows, 5:5 + cols]
    Orthogonalizer([inside], [at]).run()
    assert torch.equal(at, want)
    at.fill_(7.0)
    assert (target == 7.0).all()
    Orthogonalizer([inside], [inside]).run()
    assert torch.equal(inside, want) and torch.isnan(wide[:, :4]).all() and torch.isnan(wide[:, :, 33 + cols:]).all()
    Orthogonalizer([x[1]], [x[1]]).run()
    assert torch.equal(x[1], want[1])


def step_truth(p, g, m, h, terms, s=1.0, lr=None):
    """(p, m and the bound of p's update) in 64 bits"""
    lr = h.lr if lr is None else lr
    g = g.double().cpu() * s
    m = h.momentum * m.double().cpu() + g
    u = g + h.momentum * m if h.nesterov else m
    rows, cols = p.shape
    scale = {0: math.sqrt(max(1.0, rows / cols)), 1: 0.2 * math.sqrt(max(rows, cols)), 2: 1.0}[h.scale]
    o, off = steps_of(u, terms, eps=h.eps)
    # (m, u and lr are binary32)
    off = off + 64 * 2.0 ** -24 * float(o.norm())
    return p.double().cpu() * (1 - lr * h.weight_decay) - lr * scale * o, m, lr * scale * off


@pytest.mark.parametrize("p_type,g_type", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("nesterov,scale", [(True, "shape"), (False, "rms"), (True, "one")])
def test_steps_of_the_optimizer(p_type, g_type, nesterov, scale):
    check_steps([(2, 70, 130), (1, 200, 64), (3, 33, 33)], p_type, g_type, nesterov, scale)


@pytest.mark.parametrize("p_type,g_type", [("f32", "bf16"), ("bf16", "f32"), ("f16", "f16")])
def test_steps_of_thin_matrices(p_type, g_type):
    check_steps([(2, 40, 1000), (1, 1300, 64), (2, 250, 61), (1, 17, 201)], p_type, g_type, True, "shape")


def check_steps(shapes, p_type, g_type, nesterov, scale):
    p = [matrices_of(*s, TYPES[p_type], seed=i) * 0.05 for i, s in enumerate(shapes)]
    p[1] = p[1][0]
    grads = [[(matrices_of(*s, TYPES[g_type], seed=10 * t + i, steep=True) * 0.01) for i, s in enumerate(shapes)] for t in range(3)]
    for g in grads:
        g[1] = g[1][0]
    opt = Muon(p, grads[0], lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=scale)
    assert opt.list.c.terms == (1 if p_type == "bf16" else 2)
    for g in grads:
        opt.set_grads(g)
        before = [x.clone() for x in p], [x.clone() for x in opt.m]
        opt.step()
        for i in range(len(p)):
            whole = [x.view(-1, *x.shape[-2:]) for x in (p[i], opt.m[i], g[i], before[0][i], before[1][i])]
            for new, m, grad, old, m_old in zip(*whole):
                want, want_m, off = step_truth(old, grad, m_old, opt.h, opt.list.c.terms)
                assert ((m.double().cpu() - want_m).abs() <= 4 * 2.0 ** -24 * (want_m.abs() + grad.double().cpu().abs())).all()
                close(new, want, off + 4 * 2.0 ** -24 * float(want.norm()), i)


@pytest.mark.parametrize("rows,cols", KINDS)
def test_scaled_and_skipped_steps_and_a_rate_on_the_gpu(rows, cols):
    p, g = [matrices_of(2, rows, cols)], [matrices_of(2, rows, cols, seed=2)]
    scale, lr = torch.tensor([0.25], device=DEV), torch.tensor([0.125], dtype=torch.float64, device=DEV)
    opt = Muon(p, g, lr=9.0, weight_decay=0.1, grad_scale=scale, lr_now=lr)
    old, m_old = p[0].clone(), opt.m[0].clone()
    opt.step()
    want, want_m, off = step_truth(old[1], g[0][1], m_old[1], opt.h, 2, 0.25, 0.125)
    close(p[0][1], want, off + 4 * 2.0 ** -24 * float(want.norm()))
    for bad in (math.nan, math.inf, -math.inf):
        scale.fill_(bad)
        old, m_old = p[0].clone(), opt.m[0].clone()
        opt.step()
        assert torch.equal(p[0], old) and torch.equal(opt.m[0], m_old)
    scale.fill_(1.0)
    opt.step()
    assert torch.isfinite(p[0]).all() and not torch.equal(p[0], old)


def test_replayed_graph_and_another_stream():
    def made():
        p, g = [matrices_of(3, 200, 130), matrices_of(1, 64, 300)[0]], [matrices_of(3, 200, 130, seed=2), matrices_of(1, 64, 300, seed=3)[0]]
        return p, g, Muon(p, g, lr=0.1, weight_decay=0.01)

    p, g, opt = made()
    q, _, eager = made()
    base = [x.clone() for x in g]
    eager.set_grads(g)
    opt.step()
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for turn in range(4):
        for x, b in zip(g, base):
            x.copy_(b * (1 + turn) + turn)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(p + opt.m, q + eager.m):
            assert torch.equal(a, b), turn


def test_refusals():
    x = matrices_of(2, 8, 6)
    y = torch.empty_like(x)
    for bad in (dict(inputs=[x], outputs=[]), dict(inputs=[x.double()], outputs=[y]), dict(inputs=[x[:1]], outputs=[y]), dict(inputs=[x[0, 0]], outputs=[y[0, 0]]),
                dict(inputs=[x.transpose(1, 2)], outputs=[y.transpose(1, 2)]), dict(inputs=[x[:1].expand(2, 8, 6)], outputs=[y]),
                dict(inputs=[x], outputs=[x[:, :, :].flip(0)[:, :7]]), dict(inputs=[x.cpu()], outputs=[y]), dict(inputs=[x], outputs=[y], terms=3),
                dict(inputs=[x], outputs=[y], coefs=((3.0, 0.0, 0.0),) * 3), dict(inputs=[x], outputs=[y], coefs=()), dict(inputs=[x], outputs=[y], coefs=((1.0, 0.0, 0.0),) * 17),
                dict(inputs=[x], outputs=[y], coefs=((math.nan, 0.0, 0.0),)), dict(inputs=[x], outputs=[y], eps=-1.0),
                dict(inputs=[x.view(-1)[:48].view(1, 8, 6)], outputs=[x.view(-1)[6:54].view(1, 8, 6)])):
        with pytest.raises(cs.CsError):
            Orthogonalizer(**bad).run()
    m = torch.zeros(2, 8, 6, device=DEV)
    for bad in (dict(params=[], grads=[]), dict(params=[y], grads=[x], m=[m[:1]]), dict(params=[y], grads=[x], m=[m.half()]), dict(params=[y], grads=[y]),
                dict(params=[y], grads=[x], m=[y]), dict(params=[y], grads=[x], momentum=1.0), dict(params=[y], grads=[x], lr=-1.0),
                dict(params=[y], grads=[x], scale="area"), dict(params=[y], grads=[x], weight_decay=math.inf),
                dict(params=[y], grads=[x], lr_now=torch.ones(1, device=DEV)), dict(params=[y], grads=[x], grad_scale=torch.ones(2, device=DEV))):
        with pytest.raises(cs.CsError):
            Muon(**bad).step()
    with pytest.raises(cs.CsError, match="twice"):
        Orthogonalizer([x, x + 1], [y, y])
    with pytest.raises(cs.CsError, match="twice"):
        Muon([y, torch.empty_like(y)], [x, x], m=[m, m])
    Orthogonalizer([x, x], [y, torch.empty_like(y)]).run()                       # (what is read may be the same)
    Orthogonalizer([x[:0], x[:0]], [y[:0], y[:0]]).run()
    x, y = matrices_of(2, 70, 200), torch.zeros(2, 70, 200, device=DEV)
    opt = Muon([y], [x])
    with pytest.raises(cs.CsError, match="workspace"):
        cs.cs_muon_step(opt.h, opt.list, opt.workspace[:100])
    with pytest.raises(cs.CsError):
        cs.cs_orthogonalize(opt.h, opt.list, opt.workspace)                      # a list with moments
    with pytest.raises(cs.CsError):
        opt.set_grads([x, x])
    opt.step()                                                                   # (the list is the one that it was)
