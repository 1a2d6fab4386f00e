"""float64 definition of a beam search's selection (NumPy; nothing of the package is used), from the formulas in include/lsr_beam.h: every
continuation of every beam is listed and sorted."""
from __future__ import annotations

import numpy as np


def select(X, scores, K, temperature=1.0, finished=None, end_id=0):
    """X [B, beams, V], scores [B, beams] -> (scores float64 [B, K], beams [B, K], tokens [B, K])."""
    X, scores = np.asarray(X, np.float64), np.asarray(scores, np.float64)
    B, beams, V = X.shape
    out = np.full((B, K), -np.inf), np.zeros((B, K), np.int64), np.full((B, K), end_id, np.int64)
    for b in range(B):
        every = []                                   # (NaN first, -score, beam, -logit, token, score)
        for m in range(beams):
            s = scores[b, m]
            if s == -np.inf:
                continue
            if finished is not None and finished[b][m]:
                every.append((0 if np.isnan(s) else 1, 0.0 if np.isnan(s) else -s, m, 0.0, end_id, s))
                continue
            x = X[b, m]
            if np.isnan(s) or np.isnan(x).any() or (x == np.inf).any():
                real = [v for v in range(V) if x[v] > -np.inf]
                real.sort(key=lambda v: (-x[v], v))
                every += [(0, 0.0, m, j, v, np.nan) for j, v in enumerate((real + [end_id] * K)[:K])]
                continue
            z = x / temperature
            most = z.max()
            if most == -np.inf:
                continue
            # (the difference first: next to a mask of the type's lowest value the logarithm would be lost)
            s = s + ((z - most) - np.log(np.exp(z - most).sum()))
            every += [(1, -s[v], m, -x[v], v, s[v]) for v in range(V) if x[v] > -np.inf]
        every.sort(key=lambda c: c[:5])
        for k, c in enumerate(every[:K]):
            out[0][b, k], out[1][b, k], out[2][b, k] = c[5], c[2], c[4]
    return out


def reorder(x, parents):
    """new[b, k] = old[b, parents[b, k]], zeros where there is no such beam."""
    x = np.asarray(x)
    out = np.zeros((x.shape[0], parents.shape[1], *x.shape[2:]), x.dtype)
    for b in range(x.shape[0]):
        for k in range(parents.shape[1]):
            if 0 <= parents[b, k] < x.shape[1]:
                out[b, k] = x[b, parents[b, k]]
    return out
