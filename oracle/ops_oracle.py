"""fp64 definitions of the operators around the drafter layer, written out in numpy: layer norm and RMS
norm, token log probabilities, the AdamW step.  Test infrastructure only; the CUDA path does not import it.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ norm
def norm_fwd(kind, x, weight, bias, eps):
    """y, mean, rstd of every row; ``kind`` "layer" or "rms"; weight and bias may be None."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1) if kind == "layer" else np.zeros(x.shape[0])
    centred = x - mean[:, None]
    rstd = 1.0 / np.sqrt((centred ** 2).mean(1) + eps)
    y = centred * rstd[:, None]
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean, rstd


def norm_bwd(kind, x, weight, mean, rstd, dy):
    """dx, dweight, dbias for given statistics."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    xh = (x - np.asarray(mean, np.float64)[:, None] if kind == "layer" else x) * rstd
    u = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = u - xh * (u * xh).mean(1, keepdims=True)
    if kind == "layer":
        dx = dx - u.mean(1, keepdims=True)
    return dx * rstd, (dy * xh).sum(0), dy.sum(0)
