"""CPU oracle of the RMS norm (include/cis_norm.h): plain numpy in float64, from the formulas. Test
infrastructure only; shares no code with the HIP path."""

from __future__ import annotations

import numpy as np


def rstd(s, eps):
    s = np.asarray(s, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        return 1.0 / np.sqrt((s * s).mean(axis=-1, keepdims=True) + eps)


def forward(s, w, eps):
    """y of the rows s, which are the sums as stored."""
    with np.errstate(invalid="ignore"):
        return np.asarray(s, np.float64) * rstd(s, eps) * np.asarray(w, np.float64)


def scales(y, group):
    """[..., blocks] the scales of y's blocks of `group` columns (0: the row)."""
    n = group or y.shape[-1]
    tops = [np.abs(y[..., i:i + n]).max(axis=-1) for i in range(0, y.shape[-1], n)]
    return np.maximum(np.stack(tops, axis=-1) / 448.0, 2.0 ** -126)


def backward(dy, s, w, eps, dresidual=None):
    """(dx, dweight, sum of |dy xh|, size of what dx is a difference of)"""
    dy, s = np.asarray(dy, np.float64), np.asarray(s, np.float64)
    r = rstd(s, eps)
    xh = s * r
    g = dy * np.asarray(w, np.float64)
    mean = (g * xh).mean(axis=-1, keepdims=True)
    dx = r * (g - xh * mean)
    size = r * (np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(axis=-1, keepdims=True))
    if dresidual is not None:
        dx = dx + dresidual
        size = size + np.abs(dresidual)
    flat = (dy * xh).reshape(-1, s.shape[-1])
    return dx, flat.sum(axis=0), np.abs(flat).sum(axis=0), size
