"""float64 definitions of the operators around the head's dense logits (NumPy; nothing of the package is used).

Written from the formulas in include/lsr_distill.h, whole arrays at a time, with none of the kernels' ways of computing."""
from __future__ import annotations

import numpy as np


def quantize_rows(X):
    """(levels float64 [rows, cols], scale float64 [rows]): levels = 127 x / max|x| to nearest, ties to even."""
    X = np.asarray(X, dtype=np.float64)
    most = np.abs(X).max(axis=1)
    bad = ~np.isfinite(most)
    safe = np.where(bad | (most == 0), 1.0, most)
    levels = np.rint(np.where(np.isfinite(X), X, 0.0) * 127.0 / safe[:, None])
    levels[bad | (most == 0)] = 0.0
    return levels, np.where(bad, np.nan, most / 127.0)


def int8_matmul(A, a_scale, W, w_scale, bias=None):
    out = A.astype(np.float64) @ W.astype(np.float64).T
    out = out * np.asarray(a_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)[None, :]
    return out if bias is None else out + np.asarray(bias, np.float64)[None, :]


def top_logits(X, K, temperature):
    """(values, ids, lse): descending, equal values by ascending index, NaN first."""
    X = np.asarray(X, dtype=np.float64) + 0.0
    rank = np.where(np.isnan(X), np.inf, X)
    nan_first = np.where(np.isnan(X), 0, 1)
    ids = np.stack([np.lexsort((np.arange(X.shape[1]), -r, n)) for r, n in zip(rank, nan_first)])[:, :K]
    return np.take_along_axis(X, ids, 1), ids, log_sum_exp(X / temperature)


def log_sum_exp(x):
    m = x.max(axis=1)
    z = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        lse = z + np.log(np.exp(x - z[:, None]).sum(axis=1))
    return np.where(np.isnan(m), np.nan, np.where(np.isinf(m), m, lse))


def _teacher(ids, logits, teacher_lse, V, temperature):
    """p [N, K] (0 at padding), log p, and which entries count."""
    t = np.asarray(logits, np.float64) / temperature
    counts = (ids >= 0) & (ids < V) & (t != -np.inf)
    tm = np.where(counts, t, -np.inf)
    if teacher_lse is None:
        L = log_sum_exp(tm)
        L = np.where(np.isfinite(L), L, 0.0)
    else:
        L = np.asarray(teacher_lse, np.float64)
    logp = np.where(counts, t - L[:, None], 0.0)
    return np.where(counts, np.exp(logp), 0.0), logp, counts


def distill(H, W, bias, ids, logits, teacher_lse=None, mask=None, temperature=1.0, dloss=None):
    """{"loss", "lse"} and, with dloss, {"dH", "dW", "db", "g"}."""
    H, W, bias = (np.asarray(a, np.float64) for a in (H, W, bias))
    ids = np.asarray(ids, np.int64)
    N, V = H.shape[0], W.shape[0]
    on = np.ones(N, bool) if mask is None else np.asarray(mask) != 0
    z = (H @ W.T + bias) / temperature
    lse = log_sum_exp(z)
    p, logp, counts = _teacher(ids, logits, teacher_lse, V, temperature)
    at = np.where(counts, ids, 0)
    zt = np.take_along_axis(z, at, 1)
    used = counts & (p > 0)
    term = np.where(used, p * (logp - np.where(used, zt, 0.0) + lse[:, None]), 0.0)
    out = {"loss": np.where(on, term.sum(axis=1), 0.0), "lse": np.where(on, lse, 0.0)}
    if dloss is None:
        return out
    g = p.sum(axis=1, keepdims=True) * np.exp(z - lse[:, None])
    np.subtract.at(g, (np.arange(N)[:, None], at), np.where(used, p, 0.0))
    g *= (np.where(on, np.asarray(dloss, np.float64), 0.0) / temperature)[:, None]
    out.update(g=g, dH=g @ W, dW=g.T @ H, db=g.sum(axis=0))
    return out
