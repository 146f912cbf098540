"""The clipped policy loss, from log probabilities and from logits, against the definition in 64 bits.

Bounds, with u = 2^-24: a difference of log probabilities d is off by u |d|, its exponential r by that and 2 u of its own (the function:
less than 2 ulp); so r is off by r u (|d| + 4), and K = e^e - e - 1, by K's series or its difference, by 8 u K + u |e| |e^e - 1| (+ 4 u |e| where
it is a difference, which is below 16 u K there).  Sums are of the tokens' own values, in 64 bits, rounded once."""
import math

import pytest
import torch

import paper_1903_04488_amd as cs
from paper_1903_04488_amd.training import PolicyLoss
from test_gpu_token_logprobs import check_gradient, logits_of, reference, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TINY = 2.0 ** -148
LOW, HIGH = 0.25, 0.375                  # exact in binary32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def tokens_of(n, seed=1, spread=0.3):
    """log probabilities whose ratios are not next to a border of clipping"""
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal():
        return torch.randn(n, device=DEV, generator=gen)

    logp = -(normal() - 1.0).exp()
    d = spread * normal()
    for border in (math.log(1 - LOW), math.log(1 + HIGH)):
        d = torch.where((d - border).abs() < 1e-3, d + 4e-3, d)
    t = {"logp": logp, "entropy": normal().exp(), "old": logp - d, "ref": logp + 2 * spread * normal(), "a": normal(),
         "w": torch.rand(n, device=DEV, generator=gen) / n}
    t["w"][torch.rand(n, device=DEV, generator=gen) < 0.1] = 0.0
    t["a"][torch.rand(n, device=DEV, generator=gen) < 0.1] = 0.0
    return t


def truth(t, kl, bonus):
    """values and bounds"""
    logp, old, a, w, H = (t[k].double() for k in ("logp", "old", "a", "w", "entropy"))
    d = logp - old
    r = d.exp()
    plain, bounded = r * a, r.clamp(1 - LOW, 1 + HIGH) * a
    cut = (plain > bounded) & (w != 0)
    e = t["ref"].double() - logp
    K = torch.expm1(e) - e
    loss = w * (-torch.minimum(plain, bounded) + kl * K - bonus * H)
    g = w * (torch.where(cut, 0.0, -plain) - kl * torch.expm1(e))
    size = (plain.abs() + bounded.abs()) * U * (d.abs() + 6)
    e_k = 24 * U * K + U * e.abs() * torch.expm1(e).abs()
    r = {"loss": loss, "g_logp": g, "g_entropy": -bonus * w, "kl": w * K * (kl != 0), "cut": torch.where(cut, w, 0.0), "w": w}
    # (three more roundings for the sum and the weight)
    r["e_loss"] = w * (size + kl * e_k + 4 * U * (plain.abs() + bounded.abs() + kl * K + (bonus * H).abs())) + TINY        # (a size, whatever its sign)
    r["e_g_logp"] = w * (size + kl * U * (8 * torch.expm1(e).abs() + e.abs() * e.exp()) + 4 * U * (plain.abs() + kl * torch.expm1(e).abs())) + TINY
    r["e_g_entropy"] = 2 * U * abs(bonus) * w + TINY
    r["e_kl"] = w * (e_k + 2 * U * K) + TINY
    return r


def run(t, kl, bonus, outputs=("loss", "g_logp", "g_entropy", "sums")):
    n = len(t["logp"])
    out = {k: torch.full((4 if k == "sums" else n,), float("nan"), device=DEV) for k in outputs}
    ws = torch.empty(cs.cs_policy_workspace_bytes(n), dtype=torch.uint8, device=DEV)
    cs.cs_policy_loss(cs.CsPolicy(LOW, HIGH, kl, bonus), t["logp"], t["entropy"] if bonus else None, t["old"], t["ref"] if kl else None, t["a"],
                      t["w"], *(out.get(k) for k in ("loss", "g_logp", "g_entropy", "sums")), ws)
    return out


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1000, 1025, 8192, 8193, 300_001])
@pytest.mark.parametrize("kl,bonus", [(0.0, 0.0), (0.0625, 0.0), (0.0, 0.03125), (0.0625, 0.03125), (0.5, -0.25)])
def test_policy_loss_matches_the_definition(n, kl, bonus):
    t = tokens_of(n, seed=n)
    got, want = run(t, kl, bonus), truth(t, kl, bonus)
    for name in ("loss", "g_logp", "g_entropy"):
        within(got[name], want[name], want["e_" + name], name)
    sums = torch.stack([want["loss"].sum(), want["kl"].sum(), want["cut"].sum(), want["w"].sum()])
    bound = torch.stack([want["e_loss"].sum(), want["e_kl"].sum(), torch.zeros((), dtype=torch.float64, device=DEV), 0 * want["w"].sum()]) + U * sums.abs()
    within(got["sums"], sums, bound + TINY, "sums")


@pytest.mark.parametrize("spread", [1e-3, 1e-2, 3.0, 20.0])
def test_small_and_large_ratios(spread):
    t = tokens_of(4000, seed=3, spread=spread)
    got, want = run(t, 0.0625, 0.0), truth(t, 0.0625, 0.0)
    # e^x is beyond binary32 from x = 128 ln 2 = 88.72 on, whatever the weight makes of it: the result is within its bound or not finite
    far = (t["logp"] - t["old"] > 88.7) | (t["ref"] - t["logp"] > 88.7)
    assert bool(far.any()) == (spread == 20.0)
    for name in ("loss", "g_logp"):
        within(got[name][~far], want[name][~far], want["e_" + name][~far], name)
        fine = far & torch.isfinite(got[name])
        within(got[name][fine], want[name][fine], want["e_" + name][fine], name)


def test_borders_weights_of_zero_and_infinities():
    inf, nan = math.inf, math.nan
    # (logp, old, ref, a, w) and loss, g_logp: clip to [3/4, 11/8], kl 1
    rows = [((0.0, 0.0, 0.0, 2.0, 1.0), (-2.0, -2.0)),                           # a ratio of 1
            ((nan, nan, nan, nan, 0.0), (0.0, 0.0)),                             # left out
            ((inf, -inf, 1.0, inf, 0.0), (0.0, 0.0)),
            ((-inf, -inf, -inf, 2.0, 1.0), (-2.0, -2.0)),                        # what none allows
            ((-inf, 0.0, -inf, 2.0, 1.0), (0.0, 0.0)),                           # not any more: the ratio is 0
            ((-inf, 0.0, -inf, -2.0, 1.0), (1.5, 0.0)),                          # and clipping decides
            ((0.0, -200.0, 0.0, 2.0, 1.0), (-2.75, 0.0)),                        # a ratio beyond binary32
            ((0.0, -200.0, 0.0, 0.0, 1.0), (0.0, 0.0)),                          # without advantage
            ((0.0, -200.0, 0.0, -2.0, 1.0), (inf, inf)),                         # (the loss has no bound there)
            ((nan, 0.0, 0.0, 1.0, 1.0), (nan, nan)),
            ((0.0, 0.0, nan, 1.0, 1.0), (nan, nan)),
            ((0.0, 0.0, 0.0, nan, 1.0), (nan, nan))]
    t = dict(zip(("logp", "old", "ref", "a", "w"), torch.tensor([r[0] for r in rows], device=DEV).t().contiguous()))
    t["entropy"] = torch.zeros(len(rows), device=DEV)
    got = run(t, 1.0, 0.0)
    for name, k in (("loss", 0), ("g_logp", 1)):
        torch.testing.assert_close(got[name].cpu(), torch.tensor([r[1][k] for r in rows]), rtol=0, atol=0, equal_nan=True, msg=name)
    # at a border the ratio still counts: exp(0) against clips of 0
    one = {k: torch.zeros(2, device=DEV) for k in ("logp", "old", "ref", "entropy")} | {"a": torch.tensor([3.0, -3.0], device=DEV), "w": torch.ones(2, device=DEV)}
    g, sums = torch.empty(2, device=DEV), torch.empty(4, device=DEV)
    cs.cs_policy_loss(cs.CsPolicy(0.0, 0.0, 0.0, 0.0), one["logp"], None, one["old"], None, one["a"], one["w"], None, g, None, sums,
                      torch.empty(64, dtype=torch.uint8, device=DEV))
    assert g.tolist() == [-3.0, 3.0] and sums.tolist() == [0.0, 0.0, 0.0, 2.0]


def test_outputs_that_are_not_wanted():
    t = tokens_of(70_000, seed=4)
    whole = run(t, 0.0625, 0.03125)
    for outputs in (("loss",), ("g_logp",), ("g_entropy", "sums"), ()):
        for name, got in run(t, 0.0625, 0.03125, outputs).items():
            assert torch.equal(got, whole[name]), name


def test_gradient_against_differences():
    """(f(l + h v) - f(l - h v)) / 2h of the sum, from losses in 32 bits (off by 2^-23 of themselves, over h) and off by h^2 / 6 times the third
    derivative, which is below (r |A| + kl e^e) |v|^3; no token crosses a border within h |v|"""
    n, h, kl = 500, 2.0 ** -9, 0.25
    t = tokens_of(n, seed=5, spread=0.1)
    v = torch.randn(n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(6)).clamp(-2, 2)
    d = t["logp"] - t["old"]
    for border in (math.log(1 - LOW), math.log(1 + HIGH)):
        d = torch.where((d - border).abs() < 0.01, d + 0.02, d)
    t["old"] = t["logp"] - d
    g = run(t, kl, 0.0)["g_logp"].double()
    f = [run(t | {"logp": t["logp"] + s * h * v}, kl, 0.0)["loss"].double() for s in (1.0, -1.0)]
    moved = [(t["logp"] + s * h * v).double() for s in (1.0, -1.0)]
    slope = (f[0] - f[1]) / (2 * h)
    want = g * (moved[0] - moved[1]) / (2 * h)           # (as far as binary32 moved them)
    third = t["w"].double() * (d.double().exp() * t["a"].double().abs() + kl * (t["ref"] - t["logp"]).double().exp()) * v.double().abs() ** 3 * h * h
    noise = 16 * U * (f[0].abs() + f[1].abs() + t["w"].double() * (1 + t["a"].double().abs()) * 4) / (2 * h)
    within(slope, want, third + noise + 1e-3 * want.abs(), "slope")


def fused(x, target, t, kl, bonus, scale=1.0, in_place=False, pad=0):
    rows, vocab = x.shape
    whole = torch.full((rows, vocab + pad), -7.0, dtype=x.dtype, device=DEV)
    dx = x if in_place else whole[:, :vocab]
    logp, entropy, lse, loss = (torch.full((rows,), float("nan"), device=DEV) for _ in range(4))
    sums = torch.full((4,), float("nan"), device=DEV)
    ws = torch.empty(cs.cs_token_policy_workspace_bytes(rows, vocab), dtype=torch.uint8, device=DEV)
    cs.cs_token_policy_loss(cs.CsPolicy(LOW, HIGH, kl, bonus), x, target, t["old"], t["ref"] if kl else None, t["a"], t["w"], logp, entropy, lse,
                            loss, sums, dx, ws, scale)
    assert (whole[:, vocab:] == -7.0).all()
    return logp, entropy, lse, loss, sums, dx


def check_fused(x, target, kl, bonus, scale=1.0, pad=0, seed=7):
    """log probabilities within their bounds; losses the bits of the loss of these log probabilities, and the gradient that of its
    coefficients"""
    rows, vocab = x.shape
    r = reference(x, target, scale)
    t = tokens_of(rows, seed=seed)
    t["old"], t["ref"] = ((r["logp"].float().nan_to_num(0.0, 0.0, 0.0) + t[k] - t["logp"]).contiguous() for k in ("old", "ref"))
    logp, entropy, lse, loss, sums, dx = fused(x, target, t, kl, bonus, scale, pad=pad)
    for name, got in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        within(got, r[name], r["e_" + name], name)
    left_out = ~((target >= 0) & (target < vocab))
    again = run(t | {"logp": logp, "entropy": entropy, "w": torch.where(left_out, 0.0, t["w"])}, kl, bonus)
    assert torch.equal(loss, again["loss"])
    assert torch.equal(sums, again["sums"])
    check_gradient(dx, x, r, target, again["g_logp"], again["g_entropy"] if bonus else None, scale)
    kept = x.clone()
    in_place = fused(kept, target, t, kl, bonus, scale, in_place=True)
    assert torch.equal(in_place[-1], dx) and torch.equal(in_place[3], loss)
    return t


# rows of a wavefront, of 256, 512 and 1024 threads, of a stream, few rows and many, rows in parts
SIZES = [(1, 1), (1, 7), (5, 64), (3, 1000), (70, 1023), (300, 2048), (1100, 9001), (40, 20_000), (1030, 40_003), (2, 70_001), (1, 140_000),
         (1025, 140_001)]


@pytest.mark.parametrize("rows,vocab,dtype", [(*s, dtype) for s in SIZES for dtype in TYPES if s[0] * s[1] < 1 << 26 or dtype == "bf16"])
@pytest.mark.parametrize("kl,bonus", [(0.0625, 0.0), (0.0625, 0.03125)])
def test_from_logits(rows, vocab, dtype, kl, bonus):
    x, target = logits_of(rows, vocab, TYPES[dtype], pad=3, shift=1, seed=rows + vocab)
    if rows > 2:
        target[1], target[2] = -1, vocab
    check_fused(x, target, kl, bonus, scale=0.75, pad=5)


@pytest.mark.parametrize("rows,vocab", [(6, 500), (6, 5000), (6, 80_000), (1100, 3000)])
def test_masks(rows, vocab):
    """tokens that cannot be, an empty row, finite masks alone in a row"""
    x, target = logits_of(rows, vocab, torch.float32, seed=3)
    x[1, 1:] = -math.inf
    target[1] = 0
    x[2, : vocab // 2] = -math.inf
    target[2] = vocab - 1
    x[3] = torch.finfo(torch.float32).min
    x[4, target[4]] = -math.inf                          # the token itself cannot be
    x = x.contiguous()
    t = check_fused(x, target, 0.0, 0.03125)
    x[5] = -math.inf
    *_, dx = fused(x, target, t, 0.0, 0.03125)
    assert (dx[5] == 0).all()


def test_object_and_streams():
    x, target = logits_of(300, 9001, torch.bfloat16)
    x = x.contiguous()
    t = tokens_of(300)
    loss = PolicyLoss(300, 9001, clip=(LOW, HIGH), kl=0.0625)
    args = (target, t["old"], t["ref"], t["a"], t["w"])
    want, dx = (y.clone() for y in loss.loss(x, *args))
    assert loss.sums[3] == want[3] and abs(float(want[3]) - float(t["w"].sum())) < 1e-5
    few = loss.loss(x[:17], *(y[:17] for y in args))[1]      # (other numbers of rows have other threads: not the same bits)
    assert torch.equal(few, fused(x[:17], target[:17], {k: v[:17] for k, v in t.items()}, 0.0625, 0.0)[-1])
    assert (few.float() - dx[:17].float()).abs().max() <= 2.0 ** -7 * dx[:17].float().abs().max()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sums, again = loss.loss(x, *args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(again, dx) and torch.equal(sums, want)
    g = loss.of_logprobs(loss.logp.clone(), None, *args[1:])[1]
    assert torch.isfinite(g).all() and g.any()


def test_replayed_graph():
    x, target = logits_of(900, 70_001, torch.bfloat16)   # rows in parts: the call of several launches
    t = tokens_of(900)
    loss = PolicyLoss(900, 70_001, clip=(LOW, HIGH), kl=0.0625, entropy=0.03125)
    out = torch.empty(900, 70_001, dtype=torch.bfloat16, device=DEV)
    args = [target, t["old"].clone(), t["ref"], t["a"], t["w"]]
    loss.loss(x, *args, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss.loss(x, *args, out=out)
    for turn in range(3):
        args[1].copy_(t["old"] + 0.01 * turn)
        want = [y.clone() for y in loss.loss(x, *args)]
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(out, want[1]) and torch.equal(loss.sums, want[0])


def test_refusals():
    t = tokens_of(8)
    ws = torch.empty(cs.cs_policy_workspace_bytes(8), dtype=torch.uint8, device=DEV)
    out = [torch.empty(8, device=DEV) for _ in range(3)] + [torch.empty(4, device=DEV)]

    def call(h=None, **change):
        a = dict(logp=t["logp"], entropy=t["entropy"], old=t["old"], ref=t["ref"], a=t["a"], w=t["w"], loss=out[0], g=out[1], e=out[2],
                 sums=out[3], ws=ws) | change
        cs.cs_policy_loss(h or cs.CsPolicy(LOW, HIGH, 1.0, 1.0), *a.values())

    call()
    for bad in (dict(logp=t["logp"].double()), dict(old=t["old"][:4]), dict(ref=None), dict(entropy=None), dict(w=None), dict(a=t["a"].cpu()),
                dict(loss=t["logp"]), dict(g=out[0]), dict(sums=out[0]), dict(ws=ws[:8]), dict(ws=None), dict(old=t["old"].repeat(2)[::2]),
                dict(h=cs.CsPolicy(1.5, 0.0, 0.0, 0.0)), dict(h=cs.CsPolicy(0.0, -0.1, 0.0, 0.0)), dict(h=cs.CsPolicy(0.0, 0.0, math.nan, 0.0)),
                dict(h=cs.CsPolicy(0.0, 0.0, 0.0, math.inf))):
        with pytest.raises(cs.CsError):
            call(**bad)
    none = torch.empty(0, device=DEV)
    cs.cs_policy_loss(cs.CsPolicy(LOW, HIGH, 1.0, 1.0), *[none] * 9, out[3], torch.empty(0, dtype=torch.uint8, device=DEV))
