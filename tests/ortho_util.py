"""Plain 64-bit forms of the orthogonalised update, and how far a result of 11- or 22-bit parts may be off."""
import numpy as np

COEFS = (3.4445, -4.7750, 2.0315)


def newton_schulz(x, steps=5, coefs=COEFS, eps=1e-7):
    """(result, the X of every step) in binary64, from any matrix."""
    a, b, c = coefs
    x = np.asarray(x, dtype=np.float64)
    n = np.sqrt((x * x).sum()) + eps
    x = x / n if n > 0 else np.zeros_like(x)
    seen = [x]
    for _ in range(steps):
        if x.shape[0] > x.shape[1]:
            s = x.T @ x
            x = a * x + x @ (b * s + c * s @ s)
        else:
            s = x @ x.T
            x = a * x + (b * s + c * s @ s) @ x
        seen.append(x)
    return x, seen


def tolerance(seen, parts, out_unit, exact_start, coefs=COEFS, bound=False):
    """Frobenius norm of the error allowed to the last X, from the X of every step.

    u: half a step of what is held between the products, relative to it: 2^-11 for one fp16 part; 2^-21 for the sum of two (the second holds the first's error to 2^-11 of
    itself, 2^-22, and the dropped product of two second parts is another 2^-22). s: sums of K products in fp32, at most (K / 32 + 5) 2^-24 of the sum of magnitudes, taken as the
    product of Frobenius norms (K / 32 matrix instructions one after the other, 5 levels inside one).
    A step maps an error e of X to at most L e, L the largest |f'| for f(t) = a t + b t^3 + c t^5 over the singular values, and adds (F: Frobenius, S: spectral norm)
      of X, rounded:        L u F(X)   (not for the first X where it is held exactly)
      of A:                 (u + s) F(X)^2 at most, through b A + c A A: times (|b| + 2 |c| S(A)) S(X)
      of b A + c A A:       u F(B) + |c| s F(A)^2, times S(X)
      of the product with X: s F(B) F(X), and the final a X + ..: 2 2^-24 F.
    Errors of second order: 10% more. S(X): with `bound`, what the coefficients allow (at most 1 to begin with), without a singular value decomposition. seen may hold torch matrices."""
    a, b, c = coefs
    u = 2.0**-11 if parts == 1 else 2.0**-21
    f = lambda m: float((m * m).sum()) ** 0.5  # noqa: E731
    top = 1.0
    e = 0.0 if exact_start else u * f(seen[0])
    for i, x in enumerate(seen[:-1]):
        wide = x if x.shape[0] <= x.shape[1] else x.T
        s_x = top if bound else np.linalg.norm(wide, 2)
        t = np.linspace(0, s_x * 1.01, 2001)
        top = np.abs(a * t + b * t**3 + c * t**5).max()
        ell = np.abs(a + 3 * b * t**2 + 5 * c * t**4).max()
        s = (max(wide.shape) / 32 + 5) * 2.0**-24
        gram = wide @ wide.T
        poly = b * gram + c * gram @ gram
        e = ell * e + (ell * u * f(x) if i > 0 else 0.0)
        e += (u + s) * f(x) ** 2 * (abs(b) + 2 * abs(c) * s_x**2) * s_x
        e += (u * f(poly) + abs(c) * s * f(gram) ** 2) * s_x + s * f(poly) * f(x) + 2 * 2.0**-24 * f(seen[i + 1])
    return 1.1 * e + out_unit * f(seen[-1])


def _held(x, scale, parts):
    y = x * scale
    hi = y.half().float()
    if parts > 1:
        hi = hi + (y - hi).half().float()
    return hi / scale


def rounded(x, parts, pairs=False, steps=5, coefs=COEFS):
    """The same steps in fp32 with every matrix between the products rounded to the parts that hold it (X, A times 2^10, B times 2^8), one at a time or in pairs that
    leave X out: M = a I + B, A' = M A M, X'' = (a I + B') M X. A torch matrix, rows <= cols."""
    import torch

    a, b, c = coefs
    half = lambda m: torch.tril(m) + torch.tril(m, -1).t()  # noqa: E731
    mm = lambda p, q: p @ q.contiguous()  # noqa: E731
    x = _held((x.double() / x.double().norm()).float(), 1024.0, parts)
    i = 0
    while i < steps:
        gram = _held(half(mm(x, x.t())), 1024.0, parts)
        poly = _held(half(b * gram + c * mm(gram, gram)), 256.0, parts)
        if pairs and i + 1 < steps:
            y = _held(half(a * gram + mm(poly, gram)), 1024.0, parts)
            gram = _held(half(a * y + mm(y, poly)), 1024.0, parts)
            nxt = _held(half(b * gram + c * mm(gram, gram)), 256.0, parts)
            both = _held(half(a * poly + a * nxt + mm(nxt, poly)), 256.0, parts)
            x = a * a * x + mm(both, x)
            i += 2
        else:
            x = a * x + mm(poly, x)
            i += 1
        if i < steps:
            x = _held(x, 1024.0, parts)
    return x
