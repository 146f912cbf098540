"""Steps that are counted on the GPU, at the C boundary without one: what is refused is refused before anything is launched."""
import ctypes
import os

import pytest

import paper_1903_04488_amd as cs
from paper_1903_04488_amd import binding

F32 = 2
OK, EINVAL, EWORKSPACE = 0, -1, -2
A, B_, C, D, E, H = (0x10000000 * (i + 1) for i in range(6))
GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cs.library_path()):
        from paper_1903_04488_amd.build import build_library
        build_library()
    return cs.load_library()


def test_counting_refuses(lib):
    h = binding.CsAdamw(**GOOD)
    assert lib.cs_adamw_advance_scaled(ctypes.byref(binding.CsAdamw(**GOOD | dict(beta1=1.0))), A, None, D, B_, None) == EINVAL
    assert lib.cs_adamw_advance_scaled(ctypes.byref(h), None, None, D, B_, None) == EINVAL
    assert lib.cs_adamw_advance_scaled(ctypes.byref(h), A, None, D, None, None) == EINVAL
    assert lib.cs_adamw_advance_scaled(None, A, None, D, B_, None) == EINVAL


def test_norm_and_count_refuse(lib):
    def call(**change):
        a = dict(list=ctypes.byref(binding.CsTensorList(H, 10, 2, F32, F32, 32)), max_norm=1.0, out=A, ws=B_, ws_bytes=1 << 16,
                 h=ctypes.byref(binding.CsAdamw(**GOOD)), step=C, lr=D, coefs=E) | change
        return lib.cs_grad_norm_advance(*a.values(), None)

    for change in (dict(list=None), dict(max_norm=0.0), dict(max_norm=float("nan")), dict(out=None), dict(ws=None), dict(ws=B_ + 4), dict(h=None),
                   dict(h=ctypes.byref(binding.CsAdamw(**GOOD | dict(lr=-1.0)))), dict(step=None), dict(coefs=None), dict(out=C + 4),
                   dict(coefs=A + 4), dict(coefs=C), dict(step=B_ + 8), dict(coefs=B_ + 64), dict(lr=A), dict(lr=E + 8), dict(lr=C)):
        assert call(**change) == EINVAL, change
    assert call(ws_bytes=8) == EWORKSPACE
