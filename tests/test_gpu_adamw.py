"""AdamW over many tensors against numpy: bit for bit in binary32, operation by operation in the documented order, and against the
definition in 64 bits; moments in 8 bits code by code; the gradients' norm against 64-bit sums.

Bound against 64 bits, u = 2^-24: m and v are a sum of two products, 3u of the sum of their magnitudes; the root halves v's relative
error, the quotient adds four roundings, so the update is off by 10 u (|m| + |(1 - b1) g|) / denominator and p by that and 3 u."""
import math

import numpy as np
import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import AdamW, MomentReader, write_moments

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LENGTHS = [1, 2, 3, 4, 5, 0, 63, 255, 256, 257, 511, 1024, 4095, 4096, 4097, 20_001, 70_000]


def host(t):
    return t.detach().float().cpu().numpy()


def tensors(lengths, dtype, seed, scale=1.0, shift=0):
    """each begins `shift` values into its memory, whose rest is 77"""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    whole = [torch.full((n + shift + 9,), 77.0, dtype=dtype, device=DEV) for n in lengths]
    out = [w[shift:shift + n] for w, n in zip(whole, lengths)]
    for t in out:
        t.copy_(torch.randn(t.numel(), generator=gen, device=DEV) * scale)
    return out, whole


# ---- the documented format, in numpy ------------------------------------------------------
def encode8(x, signed):
    x = np.asarray(x, dtype=np.float32)
    n = x.size
    mag = np.zeros(-(-n // 256) * 256, dtype=np.float64)
    mag[:n] = np.abs(x)
    blocks = mag.reshape(-1, 256)
    E = np.maximum(np.where(blocks.max(1) > 0, np.floor(np.log2(np.maximum(blocks.max(1), 1e-300))) + 127, 16), 16).astype(int)
    f = 3 if signed else 4
    most = 127 if signed else 255
    unit = np.repeat(2.0 ** (E - 127.0 - 15), 256)[:n]
    a = np.abs(x).astype(np.float64) / unit
    e = np.floor(np.log2(np.maximum(a, 1e-300)))
    # the code line: e 2^f + (a / 2^e - 1) 2^f, to the nearest whole number, halves up
    line = e * 2 ** f + (a / 2.0 ** e - 1) * 2 ** f
    code = np.where(a > 0, np.clip(np.floor(line + 0.5), 0 if signed else 1, most), 0).astype(np.uint8)
    if signed:
        code = code | (np.signbit(x).astype(np.uint8) << 7)
    return code, E.astype(np.uint8)


def decode8(code, E, signed):
    code = code.astype(int)
    f = 3 if signed else 4
    c = code & 127 if signed else code
    v = np.where(c > 0, 2.0 ** ((c >> f) - 15.0) * (1 + (c % 2 ** f) / 2 ** f), 0.0) * np.repeat(2.0 ** (E.astype(float) - 127), 256)[:code.size]
    return np.where(signed & (code > 127), -v, v).astype(np.float32)


def expected(p, g, m, v, h, t, scale=None):
    """float32 arrays, every operation by itself"""
    f = np.float32
    c1, c2 = 1 / (1 - h.beta1 ** t), 1 / math.sqrt(1 - h.beta2 ** t)
    if scale is not None:
        g = g * f(scale)
    m = m * f(h.beta1) + g * f(1 - h.beta1)
    v = v * f(h.beta2) + g * g * f(1 - h.beta2)
    root = np.sqrt(v)
    p = p * f(1 - h.lr * h.weight_decay) - (m / (root * f(c2) + f(h.eps))) * f(h.lr * c1)
    return p, m, v, root


def rounded_to(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).float().numpy()


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("g_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("p_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_match_bit_for_bit(bits, p_type, g_type, shift):
    p, p_whole = tensors(LENGTHS, TYPES[p_type], 1, 0.5, shift)
    g, _ = tensors(LENGTHS, TYPES[g_type], 2, 0.01, shift)
    opt = AdamW(p, g, lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, bits=bits)
    now = [(host(a), np.zeros(a.numel(), np.float32), np.zeros(a.numel(), np.float32)) for a in p]
    for t in range(1, 4):
        for i, x in enumerate(g):
            x.mul_(-0.7 if i % 2 else 1.3)
        opt.step()
        for i, (pp, mm, vv) in enumerate(now):
            pp, mm, vv, root = expected(pp, host(g[i]), mm, vv, opt.h, t)
            pp = rounded_to(pp, TYPES[p_type])
            np.testing.assert_array_equal(host(p[i]), pp)
            if bits == 32:
                np.testing.assert_array_equal(host(opt.m[i]), mm)
                np.testing.assert_array_equal(host(opt.v[i]), vv)
            else:
                for x, codes, exps, signed in ((mm, opt.m, opt.m_exp, True), (root, opt.v, opt.v_exp, False)):
                    code, E = encode8(x, signed)
                    np.testing.assert_array_equal(codes[i].cpu().numpy(), code)
                    np.testing.assert_array_equal(exps[i].cpu().numpy(), E)
                mm = decode8(*encode8(mm, True), True)
                vv = np.square(decode8(*encode8(root, False), False))
            now[i] = pp, mm, vv
    for w, n in zip(p_whole, LENGTHS):
        assert (w[:shift] == 77).all() and (w[shift + n:] == 77).all()


def test_a_step_against_64_bits():
    lengths = [30_011, 5, 700]
    p, _ = tensors(lengths, torch.float32, 1)
    g, _ = tensors(lengths, torch.float32, 2, 0.02)
    m, _ = tensors(lengths, torch.float32, 3, 0.01)
    v = [x.square() for x in tensors(lengths, torch.float32, 4, 0.02)[0]]
    before = [[x.double().cpu().numpy() for x in t] for t in (p, g, m, v)]
    opt = AdamW(p, g, lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.05, m=m, v=v, steps=41)
    opt.step()
    h, t = opt.h, 42
    for i, (P, G, M, V) in enumerate(zip(*before)):
        M2, V2 = h.beta1 * M + (1 - h.beta1) * G, h.beta2 * V + (1 - h.beta2) * G ** 2
        den = np.sqrt(V2 / (1 - h.beta2 ** t)) + h.eps
        P2 = P * (1 - h.lr * h.weight_decay) - h.lr * (M2 / (1 - h.beta1 ** t)) / den
        size = np.abs(h.beta1 * M) + np.abs((1 - h.beta1) * G)
        assert (np.abs(host(m[i]) - M2) <= 3 * U * size).all()
        assert (np.abs(host(v[i]) - V2) <= 4 * U * V2).all()
        assert (np.abs(host(p[i]) - P2) <= 3 * U * np.abs(P) + 10 * U * h.lr * size / (1 - h.beta1 ** t) / den).all()


def test_more_tensors_than_a_launch_writes_and_shapes_kept():
    lengths = [(7 * i) % 300 for i in range(173)]
    p, _ = tensors(lengths, torch.float32, 5)
    g, _ = tensors(lengths, torch.float32, 6)
    want = [expected(host(a), host(b), host(a) * 0, host(a) * 0, cs.CsAdamw(1e-3, 0.9, 0.999, 1e-8, 0.01), 1)[0] for a, b in zip(p, g)]
    AdamW(p, g).step()
    for a, b in zip(p, want):
        np.testing.assert_array_equal(host(a), b)
    q = [torch.randn(5, 7, 11, device=DEV), torch.randn((), device=DEV)]
    opt = AdamW(q, [torch.ones_like(x) for x in q], bits=8)
    opt.step()
    assert opt.m[0].shape == q[0].shape and MomentReader(opt).read()[0][0].shape == q[0].shape


@pytest.mark.parametrize("g_type", ["f32", "bf16", "f16"])
def test_norm_and_clipping(g_type):
    p, _ = tensors(LENGTHS, torch.float32, 1)
    g, _ = tensors(LENGTHS, TYPES[g_type], 2, 0.3)
    norm = math.sqrt(sum(float(np.square(host(x).astype(np.float64)).sum()) for x in g))
    before = [host(x) for x in p]
    for max_norm in (0.5, 1e6):
        opt = AdamW(p, g, max_norm=max_norm)
        now = [host(x) for x in p]
        opt.step()
        assert float(opt.norm) == np.float32(norm)
        scale = np.float32(min(1.0, max_norm / (norm + 1e-6)))
        for a, x, b in zip(p, now, g):
            np.testing.assert_array_equal(host(a), expected(x, host(b), x * 0, x * 0, opt.h, 1, scale)[0])
    assert before[-1].size


def test_norm_of_very_large_and_very_small_gradients():
    g = [torch.full((5000,), 3e30, device=DEV), torch.full((3,), 1e-30, device=DEV)]
    out = torch.zeros(2, device=DEV)
    for some in (g, g[1:]):
        p = [torch.zeros_like(x) for x in some]
        opt = AdamW(p, some, max_norm=1.0)
        opt.step()
        want = math.sqrt(sum(float(x[0].double()) ** 2 * x.numel() for x in some))
        assert float(opt.norm) == pytest.approx(want, rel=2 * U)
    assert not out.any()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_norm_that_is_not_finite_changes_nothing(bits, bad):
    p, _ = tensors([5000, 30], torch.float32, 1)
    g, _ = tensors([5000, 30], torch.float32, 2)
    opt = AdamW(p, g, max_norm=1.0, bits=bits)
    opt.step()
    keep = [x.clone() for t in (p, opt.m, opt.v, *([opt.m_exp, opt.v_exp] if bits == 8 else [])) for x in t]
    g[1][7] = bad
    opt.step()
    assert not math.isfinite(float(opt.norm))
    now = [x for t in (p, opt.m, opt.v, *([opt.m_exp, opt.v_exp] if bits == 8 else [])) for x in t]
    assert all(torch.equal(a, b) for a, b in zip(keep, now))


# ---- moments in 8 bits --------------------------------------------------------------------
def test_every_code_is_read_as_documented():
    p = [torch.zeros(256 * 4, device=DEV)]
    code = torch.arange(256, dtype=torch.uint8, device=DEV).repeat(4)
    E = torch.tensor([16, 100, 127, 254], dtype=torch.uint8, device=DEV)
    opt = AdamW(p, [p[0].clone()], bits=8, m=[code], v=[code.clone()], m_exp=[E], v_exp=[E.clone()])
    m, root = MomentReader(opt).read()
    np.testing.assert_array_equal(host(m[0]), decode8(code.cpu().numpy(), E.cpu().numpy(), True))
    np.testing.assert_array_equal(host(root[0]), decode8(code.cpu().numpy(), E.cpu().numpy(), False))


def test_values_are_rounded_to_8_bits_as_documented():
    gen = np.random.default_rng(3)
    n = 256 * 40 + 77
    x = (gen.standard_normal(n) * np.exp(gen.standard_normal(n) * 4)).astype(np.float32)
    x[::5] = 0
    x[256:512] = 0                                            # a block of nothing
    x[512:768] *= 1e-37                                       # at the lower end
    # on and beside the boundaries between codes, in a block whose largest value is just below 2
    step = np.float32(2) ** np.arange(-20, 1)
    edge = np.concatenate([s * (1 + (np.arange(8) + 0.5) / 8) for s in step]).astype(np.float32)[:84]
    x[1024:1024 + 84], x[1110:1110 + 84] = edge, np.nextafter(edge, np.float32(0))
    x[1279] = 1.99
    root = np.abs(x)
    p = [torch.zeros(n, device=DEV)]
    opt = AdamW(p, [p[0].clone()], bits=8)
    write_moments(opt, [torch.from_numpy(x).to(DEV)], [torch.from_numpy(root).to(DEV)])
    for values, codes, exps, signed in ((x, opt.m, opt.m_exp, True), (root, opt.v, opt.v_exp, False)):
        code, E = encode8(values, signed)
        np.testing.assert_array_equal(exps[0].cpu().numpy(), E)
        np.testing.assert_array_equal(codes[0].cpu().numpy(), code)
    m, r = MomentReader(opt).read()
    m, r = host(m[0]).astype(np.float64), host(r[0]).astype(np.float64)
    assert ((r == 0) == (root == 0)).all()                    # a root that is not 0 stays that
    big = np.repeat([np.abs(np.pad(x, (0, 179)).reshape(-1, 256)).max(1)], 256).ravel()[:n]
    inside = np.abs(x) >= big * 2.0 ** -13
    assert (np.abs(m - x) <= np.abs(x) / 16 + 1e-45)[inside].all()
    assert (np.abs(r - root) <= root / 32 * (1 + 1e-9) + 1e-45)[inside & (root < big * 0.98)].all()


def test_sparse_gradients_in_8_bits_move_nothing_else():
    """a recovered update is 0 almost everywhere: parameters that never had a gradient stay where they are"""
    p = [torch.ones(10_000, device=DEV)]
    g = [torch.zeros(10_000, device=DEV)]
    g[0][::97] = 0.3
    opt = AdamW(p, g, lr=0.1, weight_decay=0.0, bits=8)
    for _ in range(5):
        opt.step()
    hit = g[0] != 0
    assert (p[0][~hit] == 1).all() and (p[0][hit] < 0.7).all()
    g[0].zero_()
    for _ in range(40):
        opt.step()
    # moments fade together; no step is longer than the rate times sqrt(1 / (1 - beta2)), which a root of 0 would allow
    assert torch.isfinite(p[0]).all() and (p[0] - 1).abs().max() < 45 * 0.1 * 2


def test_moments_that_are_not_finite_are_told_from_others():
    p, g = [torch.zeros(600, device=DEV)], [torch.zeros(600, device=DEV)]
    opt = AdamW(p, g, bits=8)
    g[0][3], g[0][300] = math.nan, 1.0
    opt.step()
    m, r = MomentReader(opt).read()
    assert m[0][3].isnan() and r[0][3].isnan()
    assert torch.isfinite(m[0][256:]).all() and float(m[0][300]) == pytest.approx(0.1, rel=1 / 16)


# ---- use ----------------------------------------------------------------------------------
def test_gradients_that_moved_and_changed_constants():
    p, _ = tensors([1000, 37], torch.float32, 1)
    g, _ = tensors([1000, 37], torch.float32, 2)
    q = [x.clone() for x in p]
    a, b = AdamW(p, g), AdamW(q, [x.clone() for x in g])
    a.step(), b.step()
    b.set_grads([x.clone() for x in g])
    a.h.lr = b.h.lr = 0.25
    a.step(), b.step()
    assert all(torch.equal(x, y) for x, y in zip(p, q))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_graph_of_steps_replays_as_steps_run(bits):
    """step number and learning rate live on the GPU"""
    p, _ = tensors([9000, 300], torch.float32, 1)
    g, _ = tensors([9000, 300], torch.float32, 2)
    start = [x.clone() for x in p]
    q, h = [x.clone() for x in p], [x.clone() for x in g]
    a, b = AdamW(p, g, max_norm=1.0, bits=bits, capturable=True), AdamW(q, h, max_norm=1.0, bits=bits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    b.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for t in range(4):
        b.h.lr = 1e-3 / (t + 1)
        a.lr_now.fill_(b.h.lr)
        for x, y in zip(g, h):
            x.mul_(1.1)
            y.mul_(1.1)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in zip((*p, *a.m, *a.v), (*q, *b.m, *b.v)):
            # (a power by the GPU's own function may be a unit off, and so may what it scales)
            if bits == 32:
                torch.testing.assert_close(x, y, rtol=4 * U, atol=1e-7)
    assert int(a.step_now) == 5 and not torch.equal(p[0], start[0])


def test_refusals():
    p, g = [torch.zeros(300, device=DEV)], [torch.zeros(300, device=DEV)]
    for bad in (dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=math.nan), dict(weight_decay=math.inf), dict(max_norm=0.0)):
        with pytest.raises(cs.CsError):
            AdamW(p, g, **bad).step()
    for make in (lambda: AdamW([], []), lambda: AdamW(p, []), lambda: AdamW(p, g, bits=16), lambda: AdamW(p, [g[0][:9]]),
                 lambda: AdamW([p[0].double()], g), lambda: AdamW([x.cpu() for x in p], g), lambda: AdamW(p, p),
                 lambda: AdamW([p[0], p[0][:0].half()], g + g), lambda: AdamW(p, g, bits=8, m=[torch.zeros(300, device=DEV)]),
                 lambda: AdamW(p, g, bits=8, m_exp=[torch.zeros(3, dtype=torch.uint8, device=DEV)]),
                 lambda: MomentReader(AdamW(p, g)), lambda: write_moments(AdamW(p, g), p, g),
                 lambda: AdamW([torch.zeros(4, 6, device=DEV).t()], [torch.zeros(6, 4, device=DEV)])):
        with pytest.raises(cs.CsError):
            make()
    opt = AdamW(p, g, bits=8)
    with pytest.raises(cs.CsError):
        cs.cs_moments_read(opt.list)                    # its p and g are no bf16 tensors
    with pytest.raises(cs.CsError, match="workspace"):
        cs.cs_grad_norm(opt.list, 1.0, torch.zeros(2, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV))
