"""How far Newton-Schulz steps on two fp16 pieces may be off, for the tests of their precision.

An entry of a product of the kernels is off by at most, in units of 2^-24 of sum |x| |y|: 4 for its operands' pieces
(2^-23 each), and 2 for each addition of the main products of 16 columns that the tensor cores round towards zero by up
to a unit (2^-23): four in sums of 64 columns (fp32 results), sixteen in sums of 256 (16-bit results); the small
products are 2^-11 of it.  So 12 or 36.  Sums of these parts are rounded to nearest, like the fp32 sums of the same
steps in fp32 products, which are off by 1 at least in the last of them.  What a product is off by goes through the
same map in both.  So a result is held to 16 (fp32) or 40 (16 bits, before its rounding) times what fp32 products are
off by on the same input, and 2^-21 of its norm for the scaling and the rounding at the end.

With the products hi lo and lo hi left out, or one piece of each matrix alone, results are off by a thousand times what
fp32 products are: 1.4e-3 to 3e-3 of the norm on these inputs against 1e-6.
"""
import numpy as np

import oracle as O

MUON = (3.4445, -4.7750, 2.0315)


def gradient(rows, cols, seed=0, strong=4, noise=0.2, size=1e-3):
    """A few strong directions over a floor of noise."""
    rng = np.random.default_rng(seed)
    k = max(1, min(strong, rows, cols))
    x = rng.standard_normal((rows, k)) @ rng.standard_normal((k, cols)) / np.sqrt(k)
    return size * (x + noise * rng.standard_normal((rows, cols)))


def fp32_steps(G, steps=5, coefficients=MUON, eps=1e-7):
    """The steps in fp32 products on the CPU."""
    a, b, c = (np.float32(v) for v in coefficients)
    X = (np.asarray(G, np.float64) / (np.linalg.norm(G) + eps)).astype(np.float32)
    tall = X.shape[0] > X.shape[1]
    X = np.ascontiguousarray(X.T if tall else X)
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return (X.T if tall else X).astype(np.float64)


def expected(G, steps=5, coefficients=MUON, sixteen=False, eps=1e-7):
    """(the result in 64 bits, how far one may be off it before its last rounding), for G as the kernels read it."""
    want = O.tuning.orthogonalize(G, steps, coefficients, eps)
    size = np.linalg.norm(want)
    return want, (40 if sixteen else 16) * np.linalg.norm(fp32_steps(G, steps, coefficients, eps) - want) + 2.0 ** -21 * size


def rounded_apart(off, want, spacing):
    """How far a result that is `off` before its rounding lies from `want` rounded: an element that is off by d rounds
    to a neighbour, u away, in a share d / u of places, and u is at most `spacing` of it.  So the squares add up to
    sum d u <= spacing |d| |want|; twice that for their scatter over the elements."""
    return (2 * spacing * off * np.linalg.norm(want)) ** 0.5 + off


def pieces(x, count=2):
    """2^12 x as fp16 pieces."""
    v = (4096.0 * x).astype(np.float32)
    hi = v.astype(np.float16).astype(np.float64)
    return hi, (v - hi).astype(np.float16).astype(np.float64) if count == 2 else 0 * hi


def product(x, y, cross=True):
    s = x[0] @ y[0]
    if cross:
        s = s + x[0] @ y[1] + x[1] @ y[0]
    return (s / 4096.0 ** 2).astype(np.float32)


def steps_on_pieces(G, steps=5, coefficients=MUON, count=2, cross=True):
    """The kernels' steps with exact sums; with one piece, or without the products of hi and lo, on request."""
    a, b, c = coefficients
    X = (G / (np.linalg.norm(G) + 1e-7)).astype(np.float32)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    one = np.eye(X.shape[0])
    for _ in range(steps):
        x = pieces(X, count)
        A = pieces(product(x, (x[0].T, x[1].T), cross), count)
        P = (c * product(A, A, cross) + b * (A[0] + A[1]) / 4096.0 + a * one).astype(np.float32)
        X = product(pieces(P, count), x, cross)
    return (X.T if tall else X).astype(np.float64)
