"""What the bounds of the Newton-Schulz tests let pass and what not, without a GPU: the arithmetic that is written down, and results that are wrong in
ways a kernel could be."""
import pytest
import torch

from newton_schulz import bounds, emulated, exact, start_of, within_bounds

COEFS = ((3.4445, -4.7750, 2.0315),) * 5


def matrix(rows, cols, steep=True):
    gen = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=gen)
    if steep:
        r = max(1, min(rows, cols) // 8)
        x += torch.randn(rows, r, generator=gen) @ torch.randn(r, cols, generator=gen) * 3
    return x


@pytest.mark.parametrize("rows,cols", [(64, 64), (64, 128), (65, 65), (250, 50), (127, 50), (16, 300), (130, 257), (5000, 33), (1, 70), (3, 5)])
@pytest.mark.parametrize("terms", [1, 2])
def test_bounds_tell_right_from_wrong(rows, cols, terms):
    u = matrix(rows, cols)
    want, whole, element = bounds(u, COEFS, terms)
    assert float(whole / want.norm()) < (4e-3 if terms == 1 else 2e-5)

    def right(x):
        return within_bounds(x, want, whole, element)

    assert right(want) and right(emulated(u, COEFS, terms)) and right(exact(u, COEFS, dtype=torch.float32))
    x, tall = start_of(u, 1e-7)
    for wrong in (torch.zeros_like(want), x.t() if tall else x, 0.9 * want, 0.99 * want, exact(u, COEFS[:4]), exact(u, COEFS[:4] + ((3.4445, -4.7750, 2.0),))):
        assert not right(wrong)
    if min(rows, cols) >= 50:                            # (of fewer directions none is small)
        assert not right(emulated(u, COEFS, terms, without=("x_low",)))
    if terms == 2:
        assert not right(emulated(u, COEFS, 2, without=("lows",))) and not right(emulated(u, COEFS, 1))
    elif (rows, cols) == (1, 70):
        assert not right(emulated(u, COEFS, 1, without=("diagonals",)))
    # a single row, column or tile of 16 that is not written
    for at in ((slice(rows - 1, rows), slice(None)), (slice(None), slice(cols - 1, cols)), (slice(0, 16), slice(0, 16))):
        lost = want.clone()
        lost[at] = 0.0
        assert not right(lost)


def test_the_emulation_with_many_bits_is_the_definition():
    """the rearranged steps (diagonals apart) in exact numbers"""
    u = matrix(40, 70)
    two = emulated(u, COEFS, 2)
    want = exact(u, COEFS)
    assert float((two - want).norm() / want.norm()) < 2e-6
    assert torch.equal(emulated(torch.zeros(3, 4), COEFS, 1), torch.zeros(3, 4, dtype=torch.float64))


@pytest.mark.parametrize("rows,cols", [(64, 64), (200, 130), (200, 300), (512, 512)])
@pytest.mark.parametrize("steep", [False, True])
def test_figures_of_one_and_two_terms(rows, cols, steep):
    """what is said of them: one term below half a step of bfloat16 (2^-9 of a result in the mean), two as binary32"""
    u = matrix(rows, cols, steep)
    want = exact(u, COEFS)

    def off(x):
        return float((x - want).norm() / want.norm())

    assert off(emulated(u, COEFS, 1)) < 2.0 ** -9 and off(emulated(u, COEFS, 2)) <= 2 * off(exact(u, COEFS, dtype=torch.float32))
