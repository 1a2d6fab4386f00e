"""float64 definitions of the head's dense logits in 8-bit floating point (NumPy; nothing of the package is used).

Written from the formulas in include/lsr_fp8.h, with none of the kernels' ways of computing: values are looked up in the table of all e4m3 numbers."""
from __future__ import annotations

import numpy as np


def e4m3_values():
    """The 127 finite values of codes 0 .. 126, ascending: 4 bits of exponent (bias 7, 0 for subnormals), 3 of mantissa."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append((8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9)
    return np.array(out)


TABLE = e4m3_values()


def nearest(x):
    """Codes of the nearest e4m3 values of |x| <= 448, ties to the even code."""
    x = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(TABLE, x), 1, 126)
    lo = hi - 1
    below, above = x - TABLE[lo], TABLE[hi] - x
    return np.where(below < above, lo, np.where(below > above, hi, np.where(lo % 2 == 0, lo, hi)))


def decode(q):
    """float64 values of e4m3 bytes."""
    q = np.asarray(q, np.uint8).astype(np.int64)
    code = q & 127
    v = np.where(code == 127, np.nan, TABLE[np.minimum(code, 126)])
    return np.where(q & 128, -v, v)


def exponent(most):
    """The smallest whole number >= -127 with most <= 448 2^e."""
    e = -127
    while most > 448.0 * 2.0 ** e:
        e += 1
    return e


def blocks(X, rows, cols):
    """(values that X stands for when held in blocks of rows x cols, exponent of every element's block)."""
    X = np.asarray(X, np.float64)
    values, exps = np.empty_like(X), np.empty(X.shape, np.int64)
    for r in range(0, X.shape[0], rows):
        for c in range(0, X.shape[1], cols):
            x = X[r:r + rows, c:c + cols]
            fine = np.isfinite(x)
            e = exponent(np.abs(np.where(fine, x, 0.0)).max())
            v = np.copysign(TABLE[nearest(np.where(fine, x, 0.0) * 2.0 ** -e)] * 2.0 ** e, x)
            values[r:r + rows, c:c + cols] = np.where(fine, v, np.nan)
            exps[r:r + rows, c:c + cols] = e
    return values, exps


def unpack(Q, exps, cols):
    """float64 values of e4m3 rows [n, >= cols] with exponents [ceil(cols / 512), n, 4]."""
    Q, exps = np.asarray(Q), np.asarray(exps).reshape(-1, np.asarray(Q).shape[0], 4).astype(np.int64)
    out = np.empty((Q.shape[0], cols))
    for b in range((cols + 127) // 128):
        part = slice(128 * b, min(cols, 128 * b + 128))
        out[:, part] = decode(Q[:, part]) * 2.0 ** (exps[b // 4, :, b % 4] - 127.0)[:, None]
    return out


def logits(H, W, bias=None):
    out = blocks(H, 1, 128)[0] @ blocks(W, 128, 128)[0].T
    return out if bias is None else out + np.asarray(bias, np.float64)


def gradients(H, W, dY):
    """(dH, dW, db)"""
    dY = np.asarray(dY, np.float64)
    return blocks(dY, 1, 128)[0] @ blocks(W, 128, 128)[0], blocks(dY, 128, 1)[0].T @ blocks(H, 128, 1)[0], dY.sum(axis=0)
