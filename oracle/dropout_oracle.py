"""Definition of dropout from a counter (NumPy and Python's own whole numbers; nothing of the package is used), from include/lsr_dropout.h."""
from __future__ import annotations

import numpy as np


def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): four 32-bit words of a counter of four words and a key of two."""
    x, k = list(counter), list(key)
    for r in range(10):
        if r:
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k[0], b % 2 ** 32, (a >> 32) ^ x[3] ^ k[1], a % 2 ** 32]
    return x


def number(i, seed, offset):
    """16-bit number of element i."""
    seed, offset, block = seed % 2 ** 64, offset % 2 ** 64, i // 8
    words = philox([block % 2 ** 32, block >> 32, offset % 2 ** 32, offset >> 32], [seed % 2 ** 32, seed >> 32])
    return (words[i % 8 // 2] >> (16 * (i % 2))) % 2 ** 16


def keep(n, p, seed, offset, first=0):
    """Whether elements first .. first + n - 1 are kept, and the factor of those that are."""
    least = int(np.rint(p * 65536))
    mask = np.array([number(i, seed, offset) >= least for i in range(first, first + n)], bool)
    return mask, (65536 / (65536 - least) if least < 65536 else 0.0)
