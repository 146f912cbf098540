"""Rows whose logits lie far from 0 (finite masks, nothing but the type's lowest value, large offsets) and their gradients by the
definition in 64 bits.  What probabilities are made of is differences of logits, so nothing
in the bounds grows with the logits themselves.

Bounds, u = 2^-24, d = z - max z, E = sum p |d|: a sum of exponentials is off by L = u (20 + n / 256 + 4 E) as for the forward
pass, and an exponent by 8 u (|d| + ln sum) through its product, difference and conversion to powers of two.  A gradient asked for later goes
by an lse in binary32 where that is below 256, which is 4 u 256 more at most."""
import numpy as np
import torch

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def far_rows(rows, vocab, dtype, seed=1):
    """rows around another offset each; the last kinds: nothing but the lowest value, it and ordinary ones, one token above it"""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.empty(rows, vocab, device=DEV).normal_(generator=gen) * 4
    lowest = torch.finfo(dtype).min
    at = [1000.0, -1000.0, 3e4, -3e4] if dtype == torch.float16 else [1000.0, -3e4, -1e9, 1e10, -1e10, 1e20, 2e38, -2e38]
    kinds = len(at) + 4
    for i in range(min(rows, kinds)):
        row = x[i::kinds]
        if i < len(at):
            row += at[i]
        elif i == len(at):
            row.fill_(lowest)
        elif i == len(at) + 1:
            row[:, ::2] = lowest
        elif i == len(at) + 2:
            row.fill_(lowest)
            row[:, vocab // 2] = 1.0
        # (the last kind: as they are)
    return x.clamp_(lowest, -lowest).to(dtype), torch.randint(0, vocab, (rows,), device=DEV, generator=gen)


def wanted(x, target, g, h, scale, later):
    """gradient, and how far off it may be"""
    scale = float(np.float32(scale))
    z = x.double() * scale
    n = z.shape[1]
    most = z.amax(1, keepdim=True)
    d = z - most
    e = d.exp()
    S = e.sum(1, keepdim=True)
    log_sum, p = S.log(), e / S
    E = torch.where(p > 0, p * d.abs(), 0.0).sum(1, keepdim=True)
    H, l = log_sum + E, torch.where(p > 0, d - log_sum, 0.0)
    hot = torch.zeros_like(p).scatter_(1, target[:, None], 1.0)
    g, h = g.double()[:, None], torch.zeros_like(S) if h is None else h.double()[:, None]
    ref = scale * (g * (hot - p) - h * p * (l + H))
    L = U * (20 + n / 256 + 4 * E)
    e_l = L + 8 * U * (l.abs() + 2 * log_sum + 1)
    if later:
        e_l = e_l + 4 * U * (most.abs() + log_sum).clamp(max=256.0)
    size = p * (g.abs() + h.abs() * (l + H).abs())
    e_H = 2 * L * (1 + E) + 4 * U * (log_sum + E)
    err = scale * (size * (e_l + 8 * U) + p * h.abs() * (e_l + e_H + 4 * U * (l.abs() + H)) + 4 * U * g.abs() * hot)
    return ref, err + HALF_ULP[x.dtype] * (ref.abs() + err) + SMALLEST[x.dtype]


def within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= bound)
    rows = bad.any(1).nonzero()[:, 0].tolist()
    assert not rows, f"{what}: {int(bad.sum())} of {bad.numel()} off, in rows {rows[:20]}, worst {float((off / bound)[bad].max()):.3g} of the bound"
