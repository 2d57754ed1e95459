"""Oracle of the 8-bit floating-point layers and of layer norm, in 64 bits with numpy.

A block (128 columns of a row, or 128 x 128 weights) shares the scale 2^e: with a = m 2^E (1 <= m < 2) the largest finite
magnitude, e = E - 8 (e4m3) or E - 15 (e5m2), one more where m > 1.75, at least -127, and 0 for a block of zeros.  A value
becomes the nearest multiple of its binade's step, ties to even; an infinity or NaN becomes NaN (e5m2 keeps infinities).
"""
from __future__ import annotations

import numpy as np

FORMATS = {"e4m3": (3, 8, -6), "e5m2": (2, 15, -14)}  # mantissa bits, exponent of the largest, of the smallest normal


def scales(x: np.ndarray, kind: str, rows: int = 1) -> np.ndarray:
    """The exponents e [ceil(T/rows)][ceil(K/128)]."""
    x = np.asarray(x, np.float64)
    T, K = x.shape
    a = np.zeros((-(-T // rows) * rows, -(-K // 128) * 128))
    a[:T, :K] = np.where(np.isfinite(x), np.abs(x), 0.0)
    a = a.reshape(a.shape[0] // rows, rows, a.shape[1] // 128, 128).max(axis=(1, 3)) if a.size else np.zeros((0, a.shape[1] // 128))
    m, e = np.frexp(a)  # 0.5 <= m < 1
    e = e - 1 - FORMATS[kind][1] + (m > 0.875)
    return np.where(a > 0, np.maximum(e, -127), 0).astype(np.int64)


def values(x: np.ndarray, kind: str, rows: int = 1) -> np.ndarray:
    """What the codes of x stand for."""
    x = np.asarray(x, np.float64)
    bits, _, low = FORMATS[kind]
    e = np.repeat(np.repeat(scales(x, kind, rows), rows, 0), 128, 1)[:x.shape[0], :x.shape[1]]
    with np.errstate(invalid="ignore"):
        v = np.ldexp(x, -e)
        g = np.maximum(np.frexp(np.where(np.isfinite(v), v, 0.0))[1] - 1, low) - bits
        q = np.ldexp(np.rint(np.ldexp(v, -g)), g)
        out = np.ldexp(q, e)
    out = np.where(np.isinf(x), x if kind == "e5m2" else np.nan, out)
    return np.where(np.isnan(x), np.nan, out)


def mask(gamma: np.ndarray, O: int, I: int) -> np.ndarray:
    return np.repeat(np.repeat(np.asarray(gamma, bool), 128, 0), 128, 1)[:O, :I]


def fc(x, W, gamma, bias=None, residual=None, relu=False, code="e4m3", coded=False, transposed=False, gate=None):
    """act(x^ W^t + b + r), gated: a block that is not kept takes no part, whatever x holds there.  ``coded``: x holds what codes stand for."""
    O, I = W.shape
    keep = mask(gamma, O, I)
    Wq = np.where(keep, values(np.where(keep, W, 0.0), "e4m3", 128), 0.0)
    xq = np.asarray(x, np.float64) if coded else values(x, code)
    if transposed:
        Wq, keep = Wq.T, keep.T
    y = np.zeros((xq.shape[0], Wq.shape[0]))
    with np.errstate(invalid="ignore"):
        for i in range(0, Wq.shape[1], 128):
            for o in range(0, Wq.shape[0], 128):
                if keep[o, i]:
                    y[:, o:o + 128] += xq[:, i:i + 128] @ Wq[o:o + 128, i:i + 128].T
        if bias is not None:
            y = y + np.asarray(bias, np.float64)
        if residual is not None:
            y = y + np.asarray(residual, np.float64)
    if relu:
        y = np.where(y < 0, 0.0, y)
    if gate is not None:
        y = np.where(np.asarray(gate) > 0, y, 0.0)
    return y


def grad_weight(dy, xq, gamma):
    """(dW, db): kept blocks' sums over the rows."""
    dy, xq = np.asarray(dy, np.float64), np.asarray(xq, np.float64)
    dW = np.where(mask(gamma, dy.shape[1], xq.shape[1]), dy.T @ xq, 0.0)
    return dW, dy.sum(0)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    x = np.asarray(x, np.float64)
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) * rstd
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_grad(dy, x, weight=None, eps=1e-5):
    """(dx, dweight, dbias) by the formula."""
    dy = np.asarray(dy, np.float64)
    h, _, rstd = layer_norm(x, None, None, eps)
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)
