"""float64 layer norm, its gradient and 8-bit layers, from their definitions
(test infrastructure only; shares no code with the HIP path)."""
from __future__ import annotations

import numpy as np

from .graphleap_ref import gelu_ref


def layer_norm_ref(x, gamma=None, beta=None, eps: float = 1e-5):
    """y = (x - mean) rstd gamma + beta over the last axis; returns (y, mean, rstd)."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    d = x - mean[..., None]
    rstd = 1.0 / np.sqrt((d * d).mean(-1) + eps)
    y = d * rstd[..., None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return y, mean, rstd


def layer_norm_backward_ref(dy, x, mean, rstd, gamma=None):
    """(dx, dgamma, dbeta) for rows x [R, C] with the statistics of the forward pass."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    rstd = np.asarray(rstd, dtype=np.float64)[..., None]
    xh = (x - np.asarray(mean, dtype=np.float64)[..., None]) * rstd
    h = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64)
    dx = rstd * (h - h.mean(-1, keepdims=True) - xh * (h * xh).mean(-1, keepdims=True))
    rows = tuple(range(x.ndim - 1))
    return dx, (dy * xh).sum(rows), dy.sum(rows)


def quantize_rows_ref(x):
    """(q, scale): q = rne(127 x / top), scale = top / 127, top the row's largest
    magnitude; a row with top < 2^-118 is zero, one that is not finite has scale NaN."""
    x = np.asarray(x, dtype=np.float64)
    top = np.abs(x).max(-1)
    zero, bad = top < 2.0 ** -118, ~np.isfinite(top)
    t = np.where(zero | bad, 1.0, top)
    q = np.rint(np.where((zero | bad)[..., None], 0.0, x) * 127.0 / t[..., None])
    scale = np.where(bad, np.nan, np.where(zero, 0.0, t / 127.0))
    return q.astype(np.int64), scale


def linear_q8_ref(q, scale, Wq, w_scale, bias=None, gelu=False, residual=None):
    """act((q Wq^T) scale w_scale + bias) + residual, the sum in whole numbers."""
    # whole numbers below 2^53: exact in float64
    y = np.asarray(q, dtype=np.float64) @ np.asarray(Wq, dtype=np.float64).T
    y = y * np.asarray(scale, dtype=np.float64)[..., None] * np.asarray(w_scale, dtype=np.float64)
    if bias is not None:
        y = y + np.asarray(bias, dtype=np.float64)
    if gelu:
        y = gelu_ref(y)
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
    return y
