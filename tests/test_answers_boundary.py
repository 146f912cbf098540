"""Losses of answers and orthogonalised momentum at the C boundary without a GPU: what is refused is refused before anything is
launched (the addresses here belong to nothing), and the structs of the binding have the header's layout."""
import ctypes
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F16, F32 = 0, 1, 2
OK, EINVAL, EWORKSPACE, EHIP = 0, -1, -2, -3
A, B_, C, D, E, F, G, H, I, J, K, L, M = (0x10000000 * (i + 1) for i in range(13))       # far apart


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cs.library_path()):
        from paper_1903_04488_amd.build import build_library
        build_library()
    return cs.load_library()


def policy(lib, h=(0.2, 0.2, 0.1, 0.1), **change):
    a = dict(rows=10, logp=A, entropy=B_, old=C, ref=D, advantage=E, weight=F, loss=G, g_logp=H, g_entropy=I, sums=J, ws=K, ws_bytes=1 << 16) | change
    return lib.cs_policy_loss(ctypes.byref(cs.CsPolicy(*h)), *a.values(), None)


def test_policy_loss_refuses(lib):
    for change in (dict(rows=-1), dict(rows=(1 << 40) + 1), dict(logp=None), dict(entropy=None), dict(old=None), dict(ref=None), dict(advantage=None),
                   dict(weight=None), dict(ws=None), dict(ws=K + 4), dict(loss=A), dict(g_logp=G + 36), dict(sums=F + 36), dict(ws=J + 8),
                   dict(g_entropy=B_ - 4), dict(h=(-0.1, 0.2, 0.0, 0.0)), dict(h=(1.1, 0.2, 0.0, 0.0)), dict(h=(0.2, math.inf, 0.0, 0.0)),
                   dict(h=(0.2, 0.2, -1.0, 0.0)), dict(h=(0.2, 0.2, 0.0, math.nan))):
        assert policy(lib, **change) == EINVAL, change
    assert policy(lib, ws_bytes=31) == EWORKSPACE
    assert policy(lib, rows=0, logp=None, ws=None, ws_bytes=0) == OK
    n = ctypes.c_size_t()
    assert lib.cs_policy_workspace_bytes(-1, ctypes.byref(n)) == EINVAL and lib.cs_policy_workspace_bytes(5, None) == EINVAL
    sizes = [cs.cs_policy_workspace_bytes(n) for n in (0, 1, 1000, 10_000, 100_000, 10_000_000)]
    assert sizes == sorted(sizes)


def token_policy(lib, h=(0.2, 0.2, 0.1, 0.1), **change):
    a = dict(logits=A, rows=4, vocab=100, stride=100, fmt=F32, scale=1.0, target=B_, old=C, ref=D, advantage=E, weight=F, logp=G, entropy=H, lse=I,
             loss=J, sums=K, dlogits=L, d_stride=100, ws=M, ws_bytes=1 << 16) | change
    return lib.cs_token_policy_loss(ctypes.byref(cs.CsPolicy(*h)), *a.values(), None)


def test_token_policy_loss_refuses(lib):
    for change in (dict(rows=-1), dict(rows=1 << 24), dict(vocab=0), dict(stride=99), dict(d_stride=99), dict(fmt=7), dict(scale=0.0), dict(scale=math.nan),
                   dict(logits=None), dict(target=None), dict(old=None), dict(ref=None), dict(advantage=None), dict(weight=None), dict(logp=None),
                   dict(entropy=None), dict(lse=None), dict(dlogits=None), dict(dlogits=A + 4), dict(dlogits=A, d_stride=101), dict(logp=F),
                   dict(loss=G), dict(sums=A + 16), dict(dlogits=C - 8), dict(ws=None), dict(ws=M + 4), dict(ws=L + 8), dict(old=L + 400), dict(h=(2.0, 0.2, 0.0, 0.0))):
        assert token_policy(lib, **change) == EINVAL, change
    assert token_policy(lib, ws_bytes=63) == EWORKSPACE
    assert token_policy(lib, rows=0, logits=None, dlogits=None, ws=None, ws_bytes=0) == OK
    n = ctypes.c_size_t()
    for rows, vocab in ((-1, 5), (1 << 24, 5), (5, 0), (5, (1 << 30) + 1)):
        assert lib.cs_token_policy_workspace_bytes(rows, vocab, ctypes.byref(n)) == EINVAL


def preference(lib, h=(0, 0, 0.1, 0.0, 0.0), **change):
    a = dict(tokens=100, pairs=3, logp=A, ref=B_, counts=C, begin=D, weight=E, loss=F, reward=G, g_logp=H, sums=I, ws=J, ws_bytes=1 << 20) | change
    return lib.cs_preference_loss(ctypes.byref(cs.CsPreference(*h)), *a.values(), None)


def test_preference_loss_refuses(lib):
    for change in (dict(tokens=-1), dict(tokens=(1 << 34) + 1), dict(pairs=-1), dict(pairs=1 << 22), dict(logp=None), dict(begin=None), dict(loss=None),
                   dict(reward=None), dict(sums=None), dict(ws=None), dict(ws=J + 4), dict(g_logp=A), dict(loss=G + 20), dict(sums=E), dict(reward=D + 48),
                   dict(g_logp=C + 50), dict(h=(3, 0, 0.1, 0.0, 0.0)), dict(h=(-1, 0, 0.1, 0.0, 0.0)), dict(h=(0, 0, 0.0, 0.0, 0.0)),
                   dict(h=(0, 0, math.nan, 0.0, 0.0)), dict(h=(0, 0, 0.1, -0.1, 0.0)), dict(h=(0, 0, 0.1, 1.1, 0.0)), dict(h=(0, 0, 0.1, 0.0, math.inf))):
        assert preference(lib, **change) == EINVAL, change
    assert preference(lib, ws_bytes=163) == EWORKSPACE
    assert preference(lib, pairs=0, begin=None, ws=None, ws_bytes=0) == OK
    assert lib.cs_preference_workspace_bytes(5, -1, ctypes.byref(ctypes.c_size_t())) == EINVAL


def stack(**change):
    a = dict(p=A, g=B_, m=C, count=2, rows=8, cols=6, p_stride=6, p_step=48, g_stride=6, g_step=48) | change
    return cs.CsMatrix(*a.values())


def build(lib, stacks, p_fmt=F32, g_fmt=F32, terms=1, memory=D, nbytes=1 << 20):
    c = cs.CsMatrixList()
    return lib.cs_matrix_list_build((cs.CsMatrix * len(stacks))(*stacks), len(stacks), p_fmt, g_fmt, terms, memory, nbytes, ctypes.byref(c), None), c


def test_matrix_list_refuses(lib):
    for change in (dict(p=None), dict(g=None), dict(p=A + 2), dict(g=B_ + 1), dict(m=C + 2), dict(count=-1), dict(rows=-1), dict(cols=(1 << 20) + 1),
                   dict(rows=40_000, cols=40_000, p_stride=40_000, g_stride=40_000, count=1), dict(p_stride=5), dict(g_stride=5), dict(p_step=47),
                   dict(g_step=0), dict(g=A), dict(g=A + 100), dict(m=A), dict(m=B_ + 380), dict(g=A, m=None, g_stride=7, g_step=56),
                   dict(p_stride=1 << 60), dict(p_step=1 << 60), dict(count=1 << 21)):
        assert build(lib, [stack(**change)])[0] == EINVAL, change
    assert build(lib, [stack(), stack(p=E, g=F, m=None)])[0] == EINVAL                    # all with moments or none
    for more in (dict(p_fmt=3), dict(g_fmt=-1), dict(terms=0), dict(terms=3), dict(memory=None), dict(memory=D + 4)):
        assert build(lib, [stack()], **more)[0] == EINVAL, more
    assert build(lib, [stack()], nbytes=100)[0] == EWORKSPACE
    n = ctypes.c_size_t()
    assert lib.cs_matrix_list_bytes(None, 1, 1, ctypes.byref(n)) == EINVAL
    rc, empty = build(lib, [stack(count=0), stack(rows=0), stack(cols=0)], memory=None, nbytes=0)
    assert rc == OK and empty.matrices == 0
    h = cs.CsMuon(0.1, 0.9, 0.0, 1e-7, 1, 0, 1, 0)
    h.coefs[0][:] = 1.5, -0.5, 0.0
    assert lib.cs_muon_step(ctypes.byref(h), ctypes.byref(empty), None, None, None, 0, None) == OK
    assert lib.cs_muon_workspace_bytes(ctypes.byref(empty), ctypes.byref(n)) == OK and n.value == 0


def test_muon_refuses(lib):
    def listed(moments):
        # (as a build fills it for two matrices in a tile of 64 each)
        return cs.CsMatrixList(D, 2, 0, 0, 0, 2, 2, 0, 2, 1 << 16, F32, F32, 1, moments, 0, 0, 1, 1, 0)

    def call(optimizer=True, c=None, ws=E, ws_bytes=1 << 20, lr=None, scale=None, **change):
        a = dict(lr=0.1, momentum=0.9, weight_decay=0.0, eps=1e-7, nesterov=1, rule=0, steps=1, reserved=0) | {k: v for k, v in change.items() if k != "coefs"}
        h = cs.CsMuon(*a.values())
        for i in range(cs.CS_MUON_MAX_STEPS):
            h.coefs[i][:] = change.get("coefs", (1.5, -0.5, 0.0))
        c = listed(1 if optimizer else 0) if c is None else c
        if optimizer:
            return lib.cs_muon_step(ctypes.byref(h), ctypes.byref(c), lr, scale, ws, ws_bytes, None)
        return lib.cs_orthogonalize(ctypes.byref(h), ctypes.byref(c), ws, ws_bytes, None)

    for change in (dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=math.nan), dict(eps=-1.0), dict(rule=3),
                   dict(rule=-1), dict(steps=0), dict(steps=17), dict(coefs=(3.0, 0.0, 0.0)), dict(coefs=(math.nan, 0.0, 0.0)), dict(coefs=(0.0, 0.0, -3.0)),
                   dict(coefs=(1.0, 100.0, -100.0)), dict(coefs=(0.0, 40.0, -39.0)), dict(c=listed(0)), dict(ws=None), dict(ws=E + 8), dict(ws=D - 256),
                   dict(scale=E + 64)):
        assert call(**change) == EINVAL, change
    assert call(optimizer=False, c=listed(1)) == EINVAL
    assert call(ws_bytes=1 << 16) == EWORKSPACE
    bad = listed(1)
    bad.full_kind = 4
    assert call(c=bad) == EINVAL


def test_structs_have_the_headers_layout(tmp_path):
    structs = {"cs_policy": cs.CsPolicy, "cs_preference": cs.CsPreference, "cs_matrix": cs.CsMatrix, "cs_matrix_list": cs.CsMatrixList, "cs_muon": cs.CsMuon}
    lines = [f'printf("%zu", sizeof({name}));' + "".join(f'printf(" %zu", offsetof({name}, {f[0]}));' for f in s._fields_) + 'printf("\\n");'
             for name, s in structs.items()]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "csketch.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    want = subprocess.check_output([str(exe)], text=True).splitlines()
    for line, (name, s) in zip(want, structs.items()):
        assert line.split() == [str(ctypes.sizeof(s))] + [str(getattr(s, f[0]).offset) for f in s._fields_], name


def test_the_package_names_what_the_binding_has():
    for name in ("cs_policy_loss", "cs_token_policy_loss", "cs_preference_loss", "cs_muon_step", "cs_orthogonalize", "MatrixList"):
        assert getattr(cs, name) is getattr(binding, name)


@pytest.mark.skipif(torch.cuda.is_available(), reason="a launch that fails, for want of a GPU")
@pytest.mark.parametrize("count,side", [(39, 70), (40, 70), (41, 70), (81, 70), (2000, 8), (300, 70)])
def test_a_list_whose_first_launch_fails_says_so(lib, count, side):
    """in a process of its own: what is written behind an array ends the process at the latest when the call returns"""
    code = f"""
import ctypes, sys
sys.path.insert(0, {ROOT!r})
import paper_1903_04488_amd as cs
n = {side * side}
stack = cs.CsMatrix({A}, {E}, {I}, {count}, {side}, {side}, {side}, n, {side}, n)
c = cs.CsMatrixList()
rc = cs.load_library().cs_matrix_list_build(ctypes.byref(stack), 1, {F32}, {F32}, 1, {M}, 1 << 30, ctypes.byref(c), None)
print("status", rc)
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.split() == ["status", str(EHIP)], (done.returncode, done.stderr[-500:])


def test_a_list_knows_its_largest_matrix(lib):
    """(by it, not by the average, it is decided who sums a matrix's squares: the plan is there also where a launch fails)"""
    def plan(*shapes):
        at = [stack(p=A + (i << 40), g=A + (1 << 50) + (i << 40), m=None, count=n, rows=rows, cols=cols, p_stride=cols, p_step=rows * cols,
                    g_stride=cols, g_step=rows * cols) for i, (n, rows, cols) in enumerate(shapes)]
        return build(lib, at, nbytes=1 << 30)[1]

    if torch.cuda.is_available():
        pytest.skip("its launches must fail")
    small, large = plan((100, 128, 128)), plan((1, 2560, 2560))
    assert small.most_pieces == 4 and large.most_pieces == large.pieces == 1600
    for mixed in (plan((1, 2560, 2560), (100, 128, 128)), plan((100, 128, 128), (1, 2560, 2560), (7, 20, 30))):
        assert mixed.most_pieces >= 1600 and mixed.pieces < 1024 * mixed.matrices
    assert plan((3, 64, 64)).most_pieces == 0
