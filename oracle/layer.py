"""What a layer does between its attention calls, from its definition in
float64 (NumPy).  Test infrastructure only.

Norm: h = x + r, y = w h / sqrt(mean(h^2) + eps).  Rows as E4M3: a group of
128 values has the scale max(max |y| / 448, 2^-60).  Product: sums over blocks
of 128 values, each times its two scales.  Rotation: pairs (a, b) of a head's
first `rot` values become (a c - b s, b c + a s).  Draw: see `draw`.
"""
from __future__ import annotations

import numpy as np

LEAST_SCALE = 2.0 ** -60


def rms_norm(x, w, eps, residual=None):
    """(y, h) of rows x [..., dim]."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + residual
    return w * h / np.sqrt((h * h).mean(-1, keepdims=True) + eps), h


def gated(x):
    """silu(a) b of the rows' halves."""
    a, b = np.split(np.asarray(x, np.float64), 2, axis=-1)
    return a / (1 + np.exp(-a)) * b


def group_scales(y):
    """Scales [groups][rows] of rows y [rows][dim]."""
    return np.stack([np.maximum(np.abs(y[:, a:a + 128]).max(1) / 448, LEAST_SCALE) for a in range(0, y.shape[1], 128)])


def linear(x, xs, w, ws):
    """(y, sum of magnitudes) of code values x [m][k], w [n][k] and their scales [blocks][m], [n blocks][blocks]."""
    m, k = x.shape
    n = w.shape[0]
    y, size = np.zeros((m, n)), np.zeros((m, n))
    for b in range(-(-k // 128)):
        at = slice(128 * b, min(k, 128 * b + 128))
        c = xs[b][:, None] * np.repeat(ws[:, b], 128)[:n]
        y += (x[:, at] @ w[:, at].T) * c
        size += (np.abs(x[:, at]) @ np.abs(w[:, at]).T) * np.abs(c)
    return y, size


def turn(x, cos_sin, pairs):
    """(rows x [N][heads][128] turned by cos_sin [N][rot], the magnitudes that were added)."""
    y, size = np.array(x, np.float64), np.abs(x).astype(np.float64)
    r = cos_sin.shape[1] // 2
    c, s = cos_sin[:, None, :r], cos_sin[:, None, r:]
    i = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if pairs else (slice(0, r), slice(r, 2 * r))
    a, b = np.array(y[..., i[0]]), np.array(y[..., i[1]])
    y[..., i[0]], y[..., i[1]] = a * c - b * s, b * c + a * s
    size[..., i[0]], size[..., i[1]] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, size


def draw(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The token of one row of logits: NaN counts as -inf, +inf as the largest fp32; -1 for a row of nothing."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, np.minimum(z, float(np.finfo(np.float32).max)))
    if not (z > -np.inf).any():
        return -1
    down = np.argsort(-z, kind="stable")  # largest first, of equal ones the lower index
    if not temperature > 0:
        return int(down[0])
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z[down] > -np.inf, np.exp((z[down] - z[down[0]]) / temperature), 0.0)
    if 0 < top_k < len(z):
        w[top_k:] = 0
    if top_p < 1:
        before = np.cumsum(w) - w
        w[1:] *= before[1:] < top_p * w.sum()
    if min_p > 0:
        w[w < min(min_p, 1.0)] = 0
    kept = np.zeros(len(z))
    kept[down] = w
    upto = np.cumsum(kept)
    u = u if u > 0 else 0.0
    return int(min(np.searchsorted(upto, u * upto[-1], side="right"), np.flatnonzero(kept)[-1]))
