"""Layer norm, token log probabilities and AdamW at the C boundary without a GPU: what is refused is refused before anything is
launched (the addresses here belong to nothing), and the structs of the binding have the header's layout."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd import binding
from paper_1903_04488_amd.training import AdamW, LayerNorm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F16, F32 = 0, 1, 2
OK, EINVAL, EWORKSPACE = 0, -1, -2
A, B_, C, D, E, F, G, H = (0x10000000 * (i + 1) for i in range(8))       # far apart


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cs.library_path()):
        from paper_1903_04488_amd.build import build_library
        build_library()
    return cs.load_library()


def norm(lib, **change):
    a = dict(x=A, rows=4, cols=64, x_stride=64, fmt=F32, weight=B_, bias=C, w_fmt=F32, eps=1e-5, y=D, y_stride=64, mean=E, rstd=F) | change
    return lib.cs_layer_norm(*a.values(), None)


def test_layer_norm_refuses(lib):
    for change in (dict(rows=-1), dict(cols=0), dict(cols=(1 << 30) + 1, x_stride=1 << 31, y_stride=1 << 31), dict(x_stride=63),
                   dict(y_stride=10), dict(fmt=3), dict(fmt=-1), dict(fmt=BF16, w_fmt=F16), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(mean=None), dict(rstd=None), dict(x=None), dict(y=None), dict(y=A + 4), dict(y=A, y_stride=65),
                   dict(weight=D + 16), dict(mean=D), dict(mean=E, rstd=E + 8), dict(rows=1 << 50, x_stride=1 << 20, y_stride=1 << 20)):
        assert norm(lib, **change) == EINVAL, change
    assert norm(lib, rows=0, x=None, y=None) == OK


def grad(lib, **change):
    a = dict(dy=A, dy_stride=64, x=B_, x_stride=64, rows=4, cols=64, fmt=F32, weight=C, w_fmt=F32, mean=D, rstd=D + 64, dx=E, dx_stride=64,
             dweight=F, dbias=F + 4096, ws=G, ws_bytes=1 << 20) | change
    return lib.cs_layer_norm_grad(*a.values(), None)


def test_layer_norm_grad_refuses(lib):
    for change in (dict(rows=-1), dict(cols=0), dict(dy_stride=1), dict(dx_stride=1), dict(fmt=9), dict(w_fmt=BF16), dict(dy=None),
                   dict(mean=None), dict(dx=A + 4), dict(dx=B_ + 256), dict(dbias=F), dict(dweight=A), dict(dbias=E), dict(ws=G + 2),
                   dict(ws=None), dict(ws=A), dict(ws=F - 64), dict(dweight=C), dict(dx=C), dict(dx=D)):
        assert grad(lib, **change) == EINVAL, change
    assert grad(lib, ws_bytes=8) == EWORKSPACE
    n = ctypes.c_size_t()
    assert lib.cs_layer_norm_grad_workspace_bytes(-1, 4, ctypes.byref(n)) == EINVAL
    assert lib.cs_layer_norm_grad_workspace_bytes(4, 0, ctypes.byref(n)) == EINVAL
    assert lib.cs_layer_norm_grad_workspace_bytes(4, 4, None) == EINVAL


def test_norm_workspace_grows_with_the_rows(lib):
    """an object made for so many rows serves fewer"""
    for cols in (1, 20, 100, 500, 1000, 2000, 5000, 12_000, 50_000):
        sizes = [cs.cs_layer_norm_grad_workspace_bytes(rows, cols) for rows in (0, 1, 2, 3, 7, 8, 100, 511, 512, 513, 5000, 100_000)]
        assert sizes == sorted(sizes)


def token(lib, **change):
    a = dict(logits=A, rows=4, vocab=100, stride=100, fmt=F32, scale=1.0, target=B_, logp=C, entropy=C + 64, lse=C + 128, top=3, top_idx=D,
             top_logp=E, ws=None, ws_bytes=0) | change
    return lib.cs_token_logprobs(*a.values(), None)


def test_token_logprobs_refuses(lib):
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1, stride=1 << 31), dict(stride=99), dict(fmt=5),
                   dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(top=-1), dict(top=65), dict(vocab=2, top=3),
                   dict(top_idx=None), dict(top_logp=None), dict(target=None), dict(logits=None), dict(lse=C), dict(logp=A + 16),
                   dict(entropy=B_), dict(top_logp=D)):
        assert token(lib, **change) == EINVAL, change
    assert token(lib, vocab=100_000, stride=100_000, ws=F, ws_bytes=10) == EWORKSPACE
    assert token(lib, vocab=100_000, stride=100_000, ws=F + 4, ws_bytes=1 << 20) == EINVAL
    assert token(lib, rows=0) == OK


def test_token_gradients_refuse(lib):
    def call(**change):
        a = dict(logits=A, rows=4, vocab=100, stride=100, fmt=F16, scale=1.0, target=B_, lse=C, entropy=C + 64, g_logp=D, g_entropy=E,
                 dlogits=F, d_stride=100) | change
        return lib.cs_token_logprobs_grad(*a.values(), None)

    for change in (dict(target=None), dict(entropy=None), dict(lse=None), dict(dlogits=None), dict(d_stride=99), dict(dlogits=A + 2),
                   dict(dlogits=A, d_stride=101), dict(dlogits=C), dict(dlogits=B_ - 100), dict(scale=-1.0)):
        assert call(**change) == EINVAL, change
    assert call(rows=0) == OK

    def loss(**change):
        a = dict(logits=A, rows=4, vocab=100, stride=100, fmt=BF16, scale=1.0, target=B_, g_logp=D, g_entropy=None, logp=C, entropy=C + 64,
                 lse=C + 128, dlogits=F, d_stride=100, ws=None, ws_bytes=0) | change
        return lib.cs_token_loss(*a.values(), None)

    for change in (dict(target=None), dict(g_logp=None), dict(logp=None), dict(entropy=None), dict(lse=None), dict(dlogits=None),
                   dict(dlogits=A + 10), dict(logp=D), dict(dlogits=C), dict(lse=F + 32), dict(dlogits=D - 64)):
        assert loss(**change) == EINVAL, change
    assert loss(rows=0) == OK


def test_token_workspace_is_small(lib):
    for rows, vocab, top in ((1, 262_144, 64), (300, 131_072, 20), (10_000, 50_000, 64), (1, 1, 1)):
        assert cs.cs_token_workspace_bytes(rows, vocab, top) <= 512 * (16 + 8 * top)
    n = ctypes.c_size_t()
    for bad in ((-1, 5, 0), (1, 0, 0), (1, 5, 6), (1, 500, 65), ((1 << 24) + 1, 5, 0)):
        assert lib.cs_token_workspace_bytes(*bad, ctypes.byref(n)) == EINVAL


def build(lib, n=(100, 5), out=True, **change):
    two = ctypes.c_void_p * 2
    a = dict(p=(A, A + 4096), p_fmt=F32, g=(B_, B_ + 4096), g_fmt=F32, m=(C, C + 4096), v=(D, D + 4096), bits=32, m_exp=None, v_exp=None,
             memory=H, bytes=1 << 16) | change
    for name in ("p", "g", "m", "v", "m_exp", "v_exp"):
        if a[name] is not None:
            a[name] = two(*a[name])
    c = binding.CsTensorList()
    return lib.cs_tensor_list_build((ctypes.c_int64 * 2)(*n), 2, *a.values(), ctypes.byref(c) if out else None, None)


def test_tensor_lists_refuse(lib):
    for change in (dict(n=(-1, 5)), dict(n=(1 << 41, 5)), dict(out=False), dict(p_fmt=3), dict(g_fmt=-1), dict(bits=16), dict(p=None), dict(m=None),
                   dict(p=(None, A)), dict(p=(A + 2, A + 4096)), dict(m=(C + 1, C + 4096)), dict(g=(A + 16, B_)), dict(v=(C + 40, D)),
                   dict(bits=8), dict(bits=8, m_exp=(E, None), v_exp=(F, F + 4)), dict(bits=8, m_exp=(C + 5, E), v_exp=(F, F + 4)),
                   dict(memory=None), dict(memory=H + 4)):
        assert build(lib, **change) == EINVAL, change
    assert build(lib, bytes=64) == EWORKSPACE
    n = ctypes.c_size_t()
    assert lib.cs_tensor_list_bytes(None, 1, ctypes.byref(n)) == EINVAL
    assert lib.cs_tensor_list_bytes(None, 0, ctypes.byref(n)) == OK and n.value == 0


def test_steps_refuse(lib):
    c = binding.CsTensorList(H, 10, 2, F32, F32, 32)
    ref = ctypes.byref(c)
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    for change in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=float("inf")), dict(weight_decay=-1.0)):
        h = binding.CsAdamw(**(good | change))
        assert lib.cs_adamw_step(ctypes.byref(h), 1, ref, None, None, None) == EINVAL
        assert lib.cs_adamw_advance(ctypes.byref(h), A, None, B_, None) == EINVAL
    h = ctypes.byref(binding.CsAdamw(**good))
    assert lib.cs_adamw_step(h, 0, ref, None, None, None) == EINVAL
    assert lib.cs_adamw_step(h, 1, None, None, None, None) == EINVAL
    assert lib.cs_adamw_step(h, 1, ctypes.byref(binding.CsTensorList(None, 10, 2, F32, F32, 32)), None, None, None) == EINVAL
    assert lib.cs_adamw_step(h, 1, ctypes.byref(binding.CsTensorList(None, 0, 0, F32, F32, 32)), None, None, None) == OK
    assert lib.cs_adamw_advance(h, None, None, B_, None) == EINVAL
    assert lib.cs_grad_norm(ref, 0.0, A, B_, 1 << 20, None) == EINVAL
    assert lib.cs_grad_norm(ref, 1.0, None, B_, 1 << 20, None) == EINVAL
    assert lib.cs_grad_norm(ref, 1.0, A, A + 4, 1 << 20, None) == EINVAL
    assert lib.cs_grad_norm(ref, 1.0, A, B_, 8, None) == EWORKSPACE
    assert lib.cs_moments_read(ref, None) == EINVAL and lib.cs_moments_write(ref, None) == EINVAL


def test_binding_structs_have_the_layout_of_the_header(tmp_path):
    lines = []
    for name, struct in (("cs_tensor_list", binding.CsTensorList), ("cs_adamw", binding.CsAdamw)):
        lines.append(f"typedef char size_{name}[sizeof({name}) == {ctypes.sizeof(struct)} ? 1 : -1];")
        lines += [f"typedef char at_{name}_{f}[offsetof({name}, {f}) == {getattr(struct, f).offset} ? 1 : -1];" for f, _ in struct._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stddef.h>\n#include \"csketch.h\"\n" + "\n".join(lines) + "\n")
    subprocess.check_call(["gcc", "-std=c99", "-pedantic-errors", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)])


def test_binding_refuses_cpu_tensors(lib):
    x, w = torch.zeros(3, 8), torch.ones(8)
    for call in (lambda: cs.cs_layer_norm(x, w, w, x), lambda: cs.cs_token_logprobs(x, None, None, None, None, None, None, None),
                 lambda: AdamW([x], [x.clone()]), lambda: LayerNorm(w, w, 3).forward(x)):
        with pytest.raises(cs.CsError):
            call()


def test_what_a_launch_has_no_threads_for(lib):
    """a workgroup of 256 for a row of logits or 4096 parameters, and fewer than 2^32 threads"""
    n = ctypes.c_size_t()
    assert lib.cs_token_workspace_bytes((1 << 24) - 1, 3, 0, ctypes.byref(n)) == OK
    assert lib.cs_token_workspace_bytes(1 << 24, 3, 0, ctypes.byref(n)) == EINVAL
    assert token(lib, rows=1 << 24) == EINVAL
    assert lib.cs_tensor_list_bytes((ctypes.c_int64 * 1)((1 << 36) - 4096), 1, ctypes.byref(n)) == OK
    assert lib.cs_tensor_list_bytes((ctypes.c_int64 * 1)(1 << 36), 1, ctypes.byref(n)) == EINVAL
