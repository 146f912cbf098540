"""Orthogonalised matrices within the errors of the arithmetic that is written down for them (the emulation in newton_schulz.py), at every size at which
another kernel begins, and the optimizer's steps with them."""
import math

import pytest
import torch

from newton_schulz import bounds, within_bounds
from paper_1903_04488_amd.training import NEWTON_SCHULZ, Muon, Orthogonalizer
from test_gpu_muon import HALF_ULP, SIZES, TYPES, matrices_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(got, x, terms, what, coefs=NEWTON_SCHULZ):
    want, whole, element = bounds(x, coefs, terms)
    d = (got.double() - want).abs()
    assert within_bounds(got, want, whole, element), (what, float(d.norm() / whole), float(d.max() / element))


@pytest.mark.parametrize("count,rows,cols", SIZES + [(1, 64, 256), (2, 64, 257), (1, 256, 64), (1, 64, 8192), (1, 64, 8193), (1, 3, 30000)])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("steep", [False, True])
def test_every_size(count, rows, cols, terms, steep):
    x = matrices_of(count, rows, cols, seed=rows + 2 * cols, steep=steep)
    out = torch.full_like(x, math.nan)
    Orthogonalizer([x], [out], terms=terms).run()
    for i in range(count):
        check(out[i], x[i], terms, (i, rows, cols))


@pytest.mark.parametrize("count,rows,cols", [(3, 50, 60), (2, 40, 900), (2, 130, 200), (2, 300, 90)])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("to", ["bf16", "f16"])
@pytest.mark.parametrize("of", list(TYPES))
def test_shorter_types_are_one_rounding(count, rows, cols, terms, of, to):
    x = matrices_of(count, rows, cols, TYPES[of], seed=5, steep=True)
    whole, short = torch.empty(x.shape, device=DEV), torch.empty(x.shape, dtype=TYPES[to], device=DEV)
    Orthogonalizer([x], [whole], terms=terms).run()
    Orthogonalizer([x], [short], terms=terms).run()
    assert torch.equal(short, whole.to(TYPES[to]))
    check(whole[-1], x[-1], terms, (rows, cols))


@pytest.mark.parametrize("coefs", [((1.5, -0.5, 0.0),) * 16, ((3.4445, -4.7750, 2.0315),), ((2.0, -1.5, 0.5), (1.875, -1.25, 0.375))])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("rows,cols", [(40, 90), (60, 700), (200, 330)])
def test_other_coefficients(coefs, terms, rows, cols):
    x = matrices_of(1, rows, cols, steep=True)
    out = torch.empty_like(x)
    Orthogonalizer([x], [out], coefs=coefs, terms=terms).run()
    check(out[0], x[0], terms, coefs[0], coefs)


@pytest.mark.parametrize("rank", [1, 4, 40])
@pytest.mark.parametrize("rows,cols", [(60, 200), (50, 2000), (150, 300)])
@pytest.mark.parametrize("terms", [1, 2])
def test_few_directions_and_next_to_nothing_else(rank, rows, cols, terms):
    """the rest is 2^-11 of them, and is raised by the steps to a tenth"""
    gen = torch.Generator(device=DEV).manual_seed(rank)
    x = torch.randn(rows, rank, device=DEV, generator=gen) @ torch.randn(rank, cols, device=DEV, generator=gen)
    x += x.norm() * 2.0 ** -11 * torch.randn(rows, cols, device=DEV, generator=gen) / math.sqrt(rows * cols)
    out = torch.empty_like(x)
    Orthogonalizer([x], [out], terms=terms).run()
    check(out, x, terms, rank)


def check_step(opt, before, grads, terms, what):
    """before: (p, m); every matrix's moment and parameters after a step"""
    h = opt.h
    mu = h.momentum
    for p, m, p_old, m_old, g in zip(opt.params, opt.m, *before, grads):
        rows, cols = p.shape[-2:]
        scale = {0: math.sqrt(max(1.0, rows / cols)), 1: 0.2 * math.sqrt(max(rows, cols)), 2: 1.0}[h.scale]
        for new, now, old, was, grad in zip(*(t.reshape(-1, rows, cols) for t in (p, m, p_old, m_old, g))):
            moment = mu * was.double() + grad.double()
            assert ((now.double() - moment).abs() <= 4 * 2.0 ** -24 * (mu * was.double().abs() + grad.double().abs())).all(), what
            u = grad.double() + mu * moment if h.nesterov else moment
            x, whole, element = bounds(u.float(), NEWTON_SCHULZ, terms, h.eps)
            kept = old.double() * (1 - h.lr * h.weight_decay)
            want = kept - h.lr * scale * x
            # binary32's: of what is kept and of the update, four roundings each, and the rounding of p
            fine = 2.0 ** -22 * (kept.abs() + h.lr * scale * x.abs())
            d = ((new.double() - want).abs() - fine - HALF_ULP[p.dtype] * want.abs() - torch.finfo(p.dtype).tiny * 2.0 ** -10).clamp(min=0)
            assert torch.isfinite(d).all() and float(d.norm()) <= h.lr * scale * float(whole) * (1 + HALF_ULP[p.dtype]), (what, float(d.norm()), h.lr * scale * float(whole))
            assert float(d.max()) <= h.lr * scale * float(element) * (1 + HALF_ULP[p.dtype]), what


def odd_rows(count, rows, cols, dtype, seed):
    """a stack whose rows begin at odd places of a wider one"""
    wide = torch.zeros(count, rows, cols + 3, dtype=dtype, device=DEV)
    inside = wide[:, :, 1:1 + cols]
    inside.copy_(matrices_of(count, rows, cols, seed=seed) * 0.05)
    return inside


def run_steps(shapes, p_type, g_type, terms, nesterov=True, scale="shape", steps=2, what=""):
    p = [odd_rows(*s, TYPES[p_type], i) for i, s in enumerate(shapes)]
    grads = [matrices_of(*s, TYPES[g_type], seed=50 + i, steep=True) * 0.01 for i, s in enumerate(shapes)]
    m = [matrices_of(*s, seed=90 + i) * 0.02 for i, s in enumerate(shapes)]
    opt = Muon(p, grads, lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=scale, m=m, terms=terms)
    for _ in range(steps):
        before = [x.clone() for x in p], [x.clone() for x in m]
        opt.step()
        check_step(opt, before, grads, terms, what)
    return opt


@pytest.mark.parametrize("p_type,g_type,terms", [("f32", "f32", 2), ("f32", "bf16", 1), ("bf16", "bf16", 1), ("bf16", "f32", 2), ("f16", "f16", 2)])
@pytest.mark.parametrize("shapes", [[(2, 60, 60), (1, 250, 30), (3, 17, 201)], [(2, 40, 1000), (1, 1300, 64)], [(2, 70, 130), (1, 200, 90), (1, 300, 300)]])
@pytest.mark.parametrize("nesterov,scale", [(True, "shape"), (False, "rms")])
def test_steps_of_the_optimizer(shapes, p_type, g_type, terms, nesterov, scale):
    run_steps(shapes, p_type, g_type, terms, nesterov, scale)
