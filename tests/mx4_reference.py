"""MXFP4 rows, the layer on them and AdamW from their definitions, in 64 bits and without the library."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(D):
    return -(-17 * (-(-D // 32)) // 16) * 16


def quantize(x):
    """x [n, D] (any float type) -> uint8 [n, row_bytes(D)]."""
    x = np.asarray(x).astype(np.float64)
    n, D = x.shape
    nb = -(-D // 32)
    p = np.zeros((n, nb, 32))
    p.reshape(n, nb * 32)[:, :D] = x
    out = np.zeros((n, row_bytes(D)), np.uint8)
    finite = np.isfinite(p).all(2)
    p = np.where(finite[..., None], p, 0.0)
    top = np.abs(p).max(2)
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    q = np.abs(p) / np.exp2(e.astype(np.float64))[..., None]
    far = np.abs(q[..., None] - MAGNITUDES)                    # exact: q is x times a power of two
    best = far.min(3, keepdims=True)
    tie = far == best
    even = tie & (np.arange(8) % 2 == 0)
    code = np.where(tie.sum(3) > 1, even.argmax(3), tie.argmax(3)).astype(np.uint8)
    code |= (np.signbit(p).astype(np.uint8) << 3)
    code = np.where(finite[..., None], code, 0).astype(np.uint8).reshape(n, nb * 32)
    out[:, :16 * nb] = code[:, 0::2] | code[:, 1::2] << 4
    out[:, 16 * nb:17 * nb] = np.where(finite, e + 127, 255)
    return out


def values(rows, D):
    """float64 [n, D] that packed rows stand for."""
    rows = np.asarray(rows)
    n, nb = rows.shape[0], -(-D // 32)
    codes = rows[:, :16 * nb]
    c = np.stack([codes & 15, codes >> 4], 2).reshape(n, nb, 32)
    s = rows[:, 16 * nb:17 * nb].astype(np.float64)
    s = np.where(s == 255, np.nan, np.exp2(s - 127))
    v = np.where(c >= 8, -1.0, 1.0) * MAGNITUDES[c & 7] * s[..., None]
    return v.reshape(n, nb * 32)[:, :D]


def adamw(p, g, m, v, t, lr, b1, b2, eps, wd):
    """One step in float64."""
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = np.sqrt(v) / np.sqrt(1 - b2 ** t) + eps
    return p - lr * wd * p - lr / (1 - b1 ** t) * m / d, m, v
