"""Which matrices of a list share memory, without a GPU: the rule against every byte of small ones."""
import random

import pytest

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.binding import _all_apart, _apart, _Place


def args(at, count, rows, cols, stride, step, name="p", written=True, index=0, size=2):
    return name, written, index, at, size, count, rows, cols, stride, step


def place(*a, **k):
    return _Place(*args(*a, **k))


def bytes_of(p):
    return {p.begin + k * p.step + r * p.pitch + e for k in range(p.count) for r in range(p.rows) for e in range(p.length)}


def test_the_rule_against_every_byte():
    rng, apart, met = random.Random(1), 0, 0
    for _ in range(4000):
        def one():
            rows, cols, count = rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 3)
            stride = cols + rng.choice([0, 0, 1, 3, 5, 10])
            step = (rows - 1) * stride + cols + rng.choice([0, 2, stride - cols, stride - cols + rows * stride]) if count > 1 else 0
            return place(2 * rng.randint(0, 60), count, rows, cols, stride, step, size=rng.choice([2, 4]))
        a, b = one(), one()
        if rng.random() < 0.5:                           # alike in all but their place
            b = place(2 * rng.randint(0, 60), a.count, a.rows, a.length // 2, a.pitch // 2, a.step // 2)
        want = not (bytes_of(a) & bytes_of(b))
        assert _apart(a, b) == _apart(b, a) == want
        spans = a.end <= b.begin or b.end <= a.begin
        apart, met = apart + (want and not spans), met + (not want)
    assert apart > 200 and met > 200


def test_parts_of_one_array():
    # columns, rows, every other row, every other matrix of a stack
    for pair in ((place(0, 1, 1000, 64, 192, 0), place(128, 1, 1000, 128, 192, 0)), (place(0, 1, 500, 64, 64, 0), place(64000, 1, 500, 64, 64, 0)),
                 (place(0, 1, 500, 64, 128, 0), place(128, 1, 500, 64, 128, 0)), (place(0, 8, 10, 64, 64, 1280), place(1280, 8, 10, 64, 64, 1280)),
                 (place(0, 4, 100, 64, 192, 19200), place(128, 4, 100, 64, 192, 19200))):
        assert _apart(*pair) and _apart(*pair[::-1])
    # a row, a column or a matrix of the other
    for pair in ((place(0, 1, 500, 64, 64, 0), place(63872, 1, 500, 64, 64, 0)), (place(0, 1, 1000, 65, 192, 0), place(128, 1, 1000, 128, 192, 0)),
                 (place(0, 8, 10, 64, 64, 640), place(1280 * 3, 1, 10, 64, 64, 0)), (place(0, 1, 1000, 192, 192, 0), place(128, 1, 1000, 64, 192, 0))):
        assert not _apart(*pair) and not _apart(*pair[::-1])


def test_who_may_share():
    p = args(0, 1, 10, 10, 10, 0)
    _all_apart([p, args(0, 1, 10, 10, 10, 0, "g", False, 0)])                                       # (its own: the library looks)
    _all_apart([p, args(1000, 1, 9, 9, 9, 0, "g", False, 0), args(1000, 1, 9, 9, 9, 0, "g", False, 1)])     # (both are read)
    for other in (args(20, 1, 10, 10, 10, 0, index=1), args(100, 1, 5, 5, 5, 0, "g", False, 1), args(198, 1, 5, 5, 5, 0, "m", True, 1)):
        with pytest.raises(cs.CsError, match="overlap"):
            _all_apart([other, p])
    # many side by side, and the last one over the first
    many = [args(128 * i, 1, 300, 64, 64 * 200, 0, index=i) for i in range(200)]
    _all_apart(many)
    with pytest.raises(cs.CsError, match=r"p\[0\] and p\[200\] overlap"):
        _all_apart(many + [args(128 * 200 * 299, 1, 1, 1, 1, 0, index=200)])
