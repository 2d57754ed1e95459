"""Oracle of root-mean-square norm, low-rank adapters beside a layer and log probabilities, in 64 bits with numpy."""
from __future__ import annotations

import numpy as np


def rms_norm(h, weight=None, eps=1e-6):
    """(y, rstd) of the residual stream h."""
    h = np.asarray(h, np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    y = h * rstd[:, None]
    return (y if weight is None else y * np.asarray(weight, np.float64)), rstd


def rms_norm_grad(dy, h, weight=None, eps=1e-6, dh=None):
    """(dx, dweight) by the formula."""
    dy = np.asarray(dy, np.float64)
    n, rstd = rms_norm(h, None, eps)
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd[:, None] * (g - n * (g * n).mean(1, keepdims=True))
    return (dx if dh is None else dx + np.asarray(dh, np.float64)), (dy * n).sum(0)


def order(x):
    """The tokens of each row by their logits, largest first, of equal ones the lower first, NaN before all."""
    x = np.where(np.isnan(x), np.inf, x), ~np.isnan(x)
    return np.lexsort((np.broadcast_to(np.arange(x[0].shape[1]), x[0].shape), -x[0], x[1]), axis=1)


def log_probs(x, tokens, top=0, scale=1.0):
    """(logp, lse, entropy, top_logp, top_tokens)."""
    x = np.asarray(x, np.float64)
    T, V = x.shape
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        z = x * scale
        m = z.max(1, keepdims=True)
        none = (m == -np.inf)[:, 0]
        d = z - np.where(none[:, None], 0.0, m)
        e = np.exp(d)
        s = e.sum(1)
        lse = np.where(none, -np.inf, m[:, 0] + np.log(s))
        lp = np.where(none[:, None], -np.inf, d - np.log(s)[:, None])
        p = np.where(none[:, None], 0.0, e / s[:, None])
        entropy = -np.where(p == 0, 0.0, p * lp).sum(1)
    tokens = np.asarray(tokens, np.int64)
    logp = np.where(tokens < 0, 0.0, np.where(tokens >= V, np.nan, lp[np.arange(T), np.clip(tokens, 0, V - 1)]))
    ids = order(x)[:, :top]
    return logp, lse, entropy, np.take_along_axis(lp, ids, 1), ids


def log_probs_grad(x, tokens, dlogp=None, dentropy=None, scale=1.0):
    x = np.asarray(x, np.float64)
    T, V = x.shape
    _, lse, h, _, _ = log_probs(x, np.full(T, -1), 0, scale)
    none = lse == -np.inf
    tokens = np.asarray(tokens, np.int64)
    dl = np.zeros(T) if dlogp is None else np.where(tokens >= 0, np.asarray(dlogp, np.float64), 0.0)
    dh = np.zeros(T) if dentropy is None else np.asarray(dentropy, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        lp = x * scale - np.where(none, 0.0, lse)[:, None]
        p = np.exp(lp)
        one = np.arange(V)[None] == tokens[:, None]
        g = dl[:, None] * (one - p) - dh[:, None] * np.where(p == 0, 0.0, p * (lp + h[:, None]))
    g = np.where(none[:, None], 0.0, scale * g)
    return np.where((tokens >= V)[:, None] & ~none[:, None], np.nan, g)


def low_rank(x, A, B, scale, which):
    """(u, what each row's adapter adds): scale A x and B u; nothing where there is no adapter."""
    x = np.asarray(x, np.float64)
    u = np.zeros((x.shape[0], A.shape[1]))
    y = np.zeros((x.shape[0], B.shape[1]))
    for n in range(A.shape[0]):
        rows = np.flatnonzero(np.asarray(which) == n)
        u[rows] = float(scale[n]) * (x[rows] @ np.asarray(A[n], np.float64).T)
        y[rows] = u[rows] @ np.asarray(B[n], np.float64).T
    return u, y


def low_rank_grad(dy, x, A, B, scale, which):
    """(dA, dB)."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    u, _ = low_rank(x, A, B, scale, which)
    v, _ = low_rank(dy, np.swapaxes(B, 1, 2), np.swapaxes(A, 1, 2), scale, which)
    dA, dB = np.zeros(A.shape), np.zeros(B.shape)
    for n in range(A.shape[0]):
        rows = np.flatnonzero(np.asarray(which) == n)
        dA[n], dB[n] = v[rows].T @ x[rows], dy[rows].T @ u[rows]
    return dA, dB
