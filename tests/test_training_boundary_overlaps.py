"""Arrays that a call writes may not meet those that it reads: refused at the C boundary, before anything is launched (the addresses
here belong to nothing)."""
import os

import pytest

import paper_1903_04488_amd as cs

F32, BF16 = 2, 0
OK, EINVAL = 0, -1
A, B_, C, D, E, F = (0x10000000 * (i + 1) for i in range(6))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cs.library_path()):
        from paper_1903_04488_amd.build import build_library
        build_library()
    return cs.load_library()


def test_layer_norm_statistics_over_weight_or_bias(lib):
    def norm(**change):
        a = dict(x=A, rows=4, cols=64, x_stride=64, fmt=F32, weight=B_, bias=C, w_fmt=F32, eps=1e-5, y=D, y_stride=64, mean=E, rstd=F) | change
        return lib.cs_layer_norm(*a.values(), None)

    for change in (dict(mean=B_), dict(mean=B_ + 63 * 4), dict(rstd=B_ - 12), dict(mean=C + 16), dict(rstd=C), dict(mean=C, bias=C, weight=None),
                   dict(mean=B_ + 63 * 2, fmt=BF16, w_fmt=BF16)):
        assert norm(**change) == EINVAL, change
