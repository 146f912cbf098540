"""Every kernel of the products in tiles, for orthogonalised matrices and for the optimizer's step, wide and tall: each test names the tiles that it means
and looks for a list that is taken in them, so that a change of the rule that picks tiles takes no kernel out of the tests unseen."""
import ctypes
import functools
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from newton_schulz import bounds, within_bounds
from paper_1903_04488_amd.training import NEWTON_SCHULZ, Orthogonalizer
from test_gpu_muon import TYPES, matrices_of
from test_gpu_muon_precision import run_steps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

SIDES = [(251, 263), (131, 701), (701, 719), (251, 1003), (499, 1001), (999, 1001), (503, 2001), (301, 5003), (131, 9001), (1001, 1703), (1999, 2029), (3001, 2999)]
COUNTS = [1, 2, 3, 4, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64]
MOST = 37_000_000                        # values of a list

# of B X: tiles of 64 x 64, 64 x 128, 128 x 128, 256 x 256
FULL = {f"B X in {name}": lambda c, k=k: c.full_kind == k for k, name in enumerate(("64 x 64", "64 x 128", "128 x 128", "256 x 256"))}
# of X X^T and A A
HALF = {"64": lambda c: c.half_kind == 0 and c.gram_slices == c.square_slices == 1, "64, X X^T in slices": lambda c: c.half_kind == 0 and c.gram_slices > 1,
        "128": lambda c: c.half_kind == 1 and c.tails == 0, "128, the last in quarters": lambda c: c.half_kind == 1 and c.tails > 0 and c.gram_slices == 1,
        "128, the last in quarters in slices": lambda c: c.half_kind == 1 and c.tails > 0 and c.gram_slices > 1 and c.square_slices > 1}
KINDS = FULL | HALF


@functools.lru_cache(None)
def plans(terms):
    """(values, shapes, list) of many lists of wide and tall matrices, the smallest first.  (Only addresses are written to a list's memory.)"""
    lib, memory = cs.load_library(), torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    some = torch.empty(MOST, dtype=torch.float32, device=DEV)
    out = []
    for n, m in SIDES:
        for count in COUNTS:
            if count * n * m > MOST:
                break
            shapes = [((count + 1) // 2, n, m)] + ([(count // 2, m, n)] if count > 1 else [])
            stacks, at = (cs.CsMatrix * len(shapes))(), some.data_ptr()
            for i, (k, rows, cols) in enumerate(shapes):
                stacks[i] = cs.CsMatrix(at, at, None, k, rows, cols, cols, rows * cols, cols, rows * cols)
                at += 4 * k * rows * cols
            c = cs.CsMatrixList()
            assert lib.cs_matrix_list_build(stacks, len(shapes), 2, 2, terms, memory.data_ptr(), memory.numel(), ctypes.byref(c), None) == 0
            out.append((count * n * m, shapes, c))
    torch.cuda.synchronize()
    return sorted(out, key=lambda x: x[0])


def shapes_in(kind, terms):
    """the smallest list that is taken in these tiles, with matrices of both directions if there is one"""
    found = [s for _, s, c in plans(terms) if KINDS[kind](c)]
    assert found, f"no list here is taken in tiles of {kind}"
    return ([s for s in found if len(s) > 1] + found)[0]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("terms", [1, 2])
def test_orthogonalized(kind, terms):
    shapes = shapes_in(kind, terms)
    xs = [matrices_of(*s, seed=i, steep=True) for i, s in enumerate(shapes)]
    outs = [torch.full_like(x, math.nan) for x in xs]
    o = Orthogonalizer(xs, outs, terms=terms)
    assert KINDS[kind](o.list.c)
    o.run()
    for x, out in zip(xs, outs):
        for i in range(len(x)):
            want, whole, element = bounds(x[i], NEWTON_SCHULZ, terms)
            d = (out[i].double() - want).abs()
            assert within_bounds(out[i], want, whole, element), (shapes, i, float(d.norm() / whole), float(d.max() / element))


# (rounded parameters are of every type and begin at odd places)
@pytest.mark.parametrize("kind", list(FULL))
@pytest.mark.parametrize("p_type,g_type,terms", [("bf16", "bf16", 1), ("f32", "f32", 1), ("f32", "bf16", 2), ("f16", "f16", 2)])
def test_steps_of_the_optimizer(kind, p_type, g_type, terms):
    shapes = shapes_in(kind, terms)
    opt = run_steps(shapes, p_type, g_type, terms, steps=1, what=shapes)
    assert KINDS[kind](opt.list.c) and opt.list.c.terms == terms


@pytest.mark.parametrize("kind", list(FULL))
@pytest.mark.parametrize("terms", [1, 2])
def test_in_place_and_short_types(kind, terms):
    shapes = shapes_in(kind, terms)
    for dtype in TYPES.values():
        xs = [matrices_of(*s, dtype, seed=i) for i, s in enumerate(shapes)]
        outs = [torch.full_like(x, math.nan) for x in xs]
        Orthogonalizer(xs, outs, terms=terms).run()
        whole = [torch.empty(x.shape, device=DEV) for x in xs]
        Orthogonalizer(xs, whole, terms=terms).run()
        Orthogonalizer(xs, xs, terms=terms).run()
        for x, out, w in zip(xs, outs, whole):
            assert torch.equal(x, out) and torch.equal(out, w.to(dtype))
