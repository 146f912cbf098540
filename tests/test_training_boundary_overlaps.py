"""Arrays that a call writes may not meet those that it reads: refused at the C boundary, before anything is launched (the addresses
here belong to nothing)."""
import ctypes
import os

import pytest

import paper_1903_04488_amd as cs
from paper_1903_04488_amd import binding

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


GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)


def test_counted_steps(lib):
    h = ctypes.byref(binding.CsAdamw(**GOOD))
    for step, lr, scale, coefs in ((A, None, None, A), (A, A, None, B_), (A, B_ + 32, None, B_), (A, None, A + 4, B_), (A, None, B_ + 36, B_),
                                   (A, None, None, A - 36)):
        assert lib.cs_adamw_advance_scaled(h, step, lr, scale, coefs, None) == EINVAL, (step, lr, scale, coefs)
        if scale is None:
            assert lib.cs_adamw_advance(h, step, lr, coefs, None) == EINVAL, (step, lr, coefs)


def test_norm_over_its_list(lib):
    """2 tensors and 10 chunks: 208 bytes"""
    c = binding.CsTensorList(C, 10, 2, F32, F32, 32)
    for out, ws in ((C, B_), (C + 204, B_), (A, C + 8), (A, C - 72), (A, A + 4)):
        assert lib.cs_grad_norm(ctypes.byref(c), 1.0, out, ws, 80, None) == EINVAL, (out, ws)
    h = ctypes.byref(binding.CsAdamw(**GOOD))
    for step, coefs in ((C + 16, E), (D, C)):
        assert lib.cs_grad_norm_advance(ctypes.byref(c), 1.0, A, B_, 80, h, step, None, coefs, None) == EINVAL
