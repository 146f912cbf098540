"""Newton-Schulz steps on a matrix: by the definition in 64 bits, and in the arithmetic that the kernels of orthogonalised matrices have (what their
products take in binary16, what they keep longer), so that a test can ask for errors of this size and not of a bound's.

emulated(): sums are exact here (binary32 in the kernels), everything is stored 2^10 times as there.  What may be left out, to see that a
test would notice:  'x_low': the lower half of X,  'diagonals': those of A and B in binary32,  'lows': all lower halves that the products take (two terms)."""
import torch

UP = 1024.0


def start_of(u, eps):
    u = u.double()
    tall = u.shape[0] > u.shape[1]
    return (u.t() if tall else u) / (torch.linalg.matrix_norm(u) + eps), tall


def exact(u, coefs, eps=1e-7, dtype=torch.float64):
    """dtype: of the products (float32: what plain products give)"""
    if not u.any():
        return u.double()
    x, tall = start_of(u, eps)
    x = x.to(dtype)
    for a, b, c in coefs:
        A = x @ x.t()
        x = a * x + (b * A + c * (A @ A)) @ x
    return (x.t() if tall else x).double()


def halves(v):
    hi = v.to(torch.float16).double()
    return hi, (v - hi).to(torch.float16).double()


def emulated(u, coefs, terms, eps=1e-7, without=(), up=UP):
    if not u.any():
        return u.double()

    def product(l, r):
        """l r of pairs (upper, lower halves)"""
        p = l[0] @ r[0]
        return p + l[0] @ r[1] + l[1] @ r[0] if terms == 2 and "lows" not in without else p

    def kept(pair, low):
        return pair[0] + pair[1] if low else pair[0]

    x, tall = start_of(u, eps)
    x = x.float().double() * up
    for a, b, c in coefs:
        X = halves(x)
        x_t = tuple(v.t().contiguous() for v in X)
        A = product(X, x_t) / up ** 2
        d = A.diagonal().float().double()
        if "diagonals" in without:
            d = halves(d * up)[0] / up
        A0 = halves((A - torch.diag(A.diagonal())) * up)
        AA = product(A0, A0) / up ** 2
        low = terms == 2 and "lows" not in without
        B = (c * (d[:, None] + d[None, :]) + b) * kept(A0, low) / up + c * AA
        e = (b * d + c * (d * d + AA.diagonal())).float().double()
        if "diagonals" in without:
            e = halves(e * up)[0] / up
        B0 = halves((B - torch.diag(B.diagonal())) * up)
        x = (a + e)[:, None] * kept(X, "x_low" not in without) + product(B0, X) / up
        x = x.float().double()
    x = x / up
    return x.t() if tall else x


def bounds(u, coefs, terms, eps=1e-7):
    """(the result in 64 bits, how far off the whole may be in the 2-norm, and a single element).

    The kernels' roundings to binary16 are the emulation's, but for values that binary32's sums move past a tie and, of thin matrices, a first
    product of numbers that are scaled otherwise: errors of the same size, so twice the emulation's.  Of few directions or few values an error is a
    sum of few roundings, which may be next to nothing in one emulation by luck and not in a kernel that takes one tie otherwise: there its size is the
    largest of eight emulations at other scales (2^(k/8) of the first: other roundings), and a tie beside it: a step of binary16, 2^-11 of the largest
    value at most.  What binary32 adds is what plain products in binary32 are off by, up to the order of their sums: four times that, and
    eight times of few.  Of a single element the emulation's largest, three times."""
    want = exact(u, coefs, eps)
    few = min(u.shape) < 16 or u.numel() < 4096
    halves_off = [emulated(u, coefs, terms, eps, up=UP * 2.0 ** (k / 8)) - want for k in range(8 if few else 1)]
    whole, element = max(d.norm() for d in halves_off), max(d.abs().max() for d in halves_off)
    single = exact(u, coefs, eps, torch.float32) - want
    if few:
        step = 2.0 ** (-11 * terms) * want.abs().max()
        whole, element = whole + step, element + step
    tiny = 2.0 ** -20 * want.abs().max()
    return want, 2 * whole + (8 if few else 4) * single.norm() + tiny, 3 * element + 8 * single.abs().max() + tiny


def within_bounds(got, want, whole, element, rounded=0.0):
    """rounded: half a step of the type that got has been rounded to, relative"""
    d = ((got.double() - want).abs() - rounded * want.abs()).clamp(min=0)
    return bool(torch.isfinite(d).all()) and bool(d.norm() <= whole) and bool(d.max() <= element)
