"""Hidden rows in 8 bits and the layers on them from their definitions, in 64 bits and without the library."""
import math

import numpy as np

BLOCK, MOST, LEAST_E, MOST_E = 128, 448.0, -117, 119
# the magnitudes of codes 0 .. 126: four bits of exponent with bias 7, three of fraction
MAGNITUDES = np.array([c * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])


def code_bytes(D):
    return -(-D // 16) * 16


def row_bytes(D):
    return code_bytes(D) + -(-(-(-D // BLOCK)) // 16) * 16


def _codes(q):
    """The nearest code to each q, |q| at most 448 or beyond: ties to the even code, 448 above."""
    a = np.abs(q)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 126)
    lo = hi - 1
    up, down = MAGNITUDES[hi] - a, a - MAGNITUDES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    return code | (np.signbit(q).astype(np.uint8) << 7)


def quantize(x):
    """x [n, D] (any float type) -> uint8 [n, row_bytes(D)]."""
    x = np.asarray(x).astype(np.float64)
    n, D = x.shape
    nb, cb = -(-D // BLOCK), code_bytes(D)
    out = np.zeros((n, row_bytes(D)), np.uint8)
    for b in range(nb):
        p = x[:, b * BLOCK:(b + 1) * BLOCK]
        fine = np.isfinite(p)
        p = np.where(fine, p, 0.0)
        top = np.abs(p).max(1)
        e = np.full(n, LEAST_E)
        while True:
            small = (MOST * np.exp2(e.astype(np.float64)) < top) & (e < MOST_E)
            if not small.any():
                break
            e += small
        c = np.where(fine, _codes(p / np.exp2(e.astype(np.float64))[:, None]), 0x7F)
        out[:, b * BLOCK:b * BLOCK + p.shape[1]] = c
        out[:, cb + b] = e + 127
    return out


def values(rows, D):
    """float64 [n, D] that rows stand for."""
    rows = np.asarray(rows)
    c = rows[:, :D]
    table = np.append(MAGNITUDES, np.nan)
    v = np.where(c >= 128, -1.0, 1.0) * table[c & 127]
    s = rows[:, code_bytes(D) + np.arange(D) // BLOCK].astype(np.float64)
    return v * np.where(s == 255, np.nan, np.exp2(s - 127))


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(name, g):
    """act(g), act'(g), a bound of |act'|, one of |act''|, and how far the two computed in fp32 may be from these for the same g.

    Each operation is off by at most half a step, 2^-24 of its result, but the hardware's exponential and reciprocal by a whole one and
    the library's erfc by a few.  The argument of an exponential, off by 3 such of itself, moves it by that much times itself."""
    u = 2.0 ** -23
    if name == "gelu":
        p = 0.5 * _erfc(-g / np.sqrt(2.0))
        phi = np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
        f, d = g * p, p + g * phi
        return f, d, 1.13, 0.8, np.abs(f) * (g * g * 2 + 10) * u + 1e-37, (p + np.abs(g) * phi) * (g * g * 2 + 12) * u + 1e-37
    with np.errstate(over="ignore"):
        s, r = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    rel = (2 * np.abs(g) + 8) * u
    if name == "silu":
        return g * s, s * (1 + g * r), 1.1, 0.5, np.abs(g * s) * rel + 1e-36, s * (1 + np.abs(g) * r) * rel + 1e-36
    return s, s * r, 0.25, 0.1, s * rel + 1e-36, s * r * rel + 1e-36


def sums(x, w, bits=32):
    """x w^T and how far it may be off: K terms, each addition in fp32 off by at most 2^-23 of what it adds (cut off, not rounded).
    For results of 16 bits the terms of eight columns are first cut off at 2^-13 of the power of two of the largest of them: by less than
    8 times 2^-13 of that term, over all columns by less than 2^-10 of the sum of all terms' magnitudes."""
    size = np.abs(x) @ np.abs(w).T
    return x @ w.T, (x.shape[1] * 2.0 ** -23 + (2.0 ** -10 if bits == 16 else 0.0)) * size


def gated(x, wg, wu, name, bits=32):
    """The gated layer's values and how far they may be off before they are rounded to their type."""
    g, eg = sums(x, wg, bits)
    u, eu = sums(x, wu, bits)
    f, _, l1, _, bf, _ = activation(name, g)
    bf = bf + l1 * eg
    return f * u, np.abs(u) * bf + np.abs(f) * eu + bf * eu + np.abs(f * u) * 2.0 ** -23


def gated_grad(x, wg, wu, dy, name, bits=32):
    """[dG | dU] and how far they may be off."""
    g, eg = sums(x, wg, bits)
    u, eu = sums(x, wu, bits)
    f, d, l1, l2, bf, bd = activation(name, g)
    bf, bd = bf + l1 * eg, bd + l2 * eg
    dg, du = dy * u * d, dy * f
    a = np.abs(dy)
    return (np.concatenate([dg, du], 1),
            np.concatenate([a * (np.abs(u) * bd + np.abs(d) * eu + eu * bd) + np.abs(dg) * 2.0 ** -22, a * bf + np.abs(du) * 2.0 ** -23], 1))
