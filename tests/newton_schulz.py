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


def emulated(u, coefs, terms, eps=1e-7, without=()):
    if not u.any():
        return u.double()

    def product(l, r):
        """l r of pairs (upper, lower halves)"""
        p = l[0] @ r[0]
        return p + l[0] @ r[1] + l[1] @ r[0] if terms == 2 and "lows" not in without else p

    def kept(pair, low):
        return pair[0] + pair[1] if low else pair[0]

    x, tall = start_of(u, eps)
    x = x.float().double() * UP
    for a, b, c in coefs:
        X = halves(x)
        x_t = tuple(v.t().contiguous() for v in X)
        A = product(X, x_t) / UP ** 2
        d = A.diagonal().float().double()
        if "diagonals" in without:
            d = halves(d * UP)[0] / UP
        A0 = halves((A - torch.diag(A.diagonal())) * UP)
        AA = product(A0, A0) / UP ** 2
        low = terms == 2 and "lows" not in without
        B = (c * (d[:, None] + d[None, :]) + b) * kept(A0, low) / UP + c * AA
        e = (b * d + c * (d * d + AA.diagonal())).float().double()
        if "diagonals" in without:
            e = halves(e * UP)[0] / UP
        B0 = halves((B - torch.diag(B.diagonal())) * UP)
        x = (a + e)[:, None] * kept(X, "x_low" not in without) + product(B0, X) / UP
        x = x.float().double()
    x = x / UP
    return x.t() if tall else x


def bounds(u, coefs, terms, eps=1e-7):
    """(the result in 64 bits, how far off the whole may be in the 2-norm, and a single element).

    The kernels' roundings to binary16 are the emulation's, but for values that binary32's sums move past a tie and, of thin matrices, a first
    product of numbers that are scaled otherwise: errors of the same size, so twice the emulation's.  What binary32 adds is what plain
    products in binary32 are off by, up to the order of their sums: four times that.  Of a single element the emulation's largest, three times."""
    want = exact(u, coefs, eps)
    half, single = emulated(u, coefs, terms, eps) - want, exact(u, coefs, eps, torch.float32) - want
    tiny = 2.0 ** -20 * want.abs().max()
    return (want, 2 * half.norm() + 4 * single.norm() + tiny, 3 * half.abs().max() + 8 * single.abs().max() + tiny)


def within_bounds(got, want, whole, element, rounded=0.0):
    """rounded: half a step of the type that got has been rounded to, relative"""
    d = ((got.double() - want).abs() - rounded * want.abs()).clamp(min=0)
    return bool(torch.isfinite(d).all()) and bool(d.norm() <= whole) and bool(d.max() <= element)
