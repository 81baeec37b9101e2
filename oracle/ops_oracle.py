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


# ------------------------------------------------------------------ token log probabilities
def token_logprobs(logits, tokens, scale, k):
    """logprob, lse, entropy, top log probabilities, top ids of every row; one row at a time, by the cases
    that the header lists (token -1: no token; rows of -inf; rows with NaN or +inf)."""
    rows, vocab = logits.shape
    lp, lse, H = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    top, ids = np.zeros((rows, k)), np.full((rows, k), -1, np.int64)
    for r in range(rows):
        x = np.asarray(logits[r], np.float64)
        if np.isnan(x).any() or np.isposinf(x).any():
            lse[r] = H[r] = np.nan
            lp[r] = 0.0 if tokens[r] == -1 else np.nan
            top[r] = np.nan
            continue
        order = np.lexsort((np.arange(vocab), -x))[:k]      # by value, then by id
        ids[r] = order
        s = x * scale
        m = s.max()
        if np.isneginf(m):
            lse[r], H[r] = -np.inf, 0.0
            lp[r] = 0.0 if tokens[r] == -1 else -np.inf
            top[r] = -np.inf
        else:
            # differences to the maximum first: at 1e38, 64 bits have no room for a log of the vocabulary either
            t = s - m
            log_sum = np.log(np.exp(t).sum())
            lse[r] = m + log_sum
            logp = t - log_sum
            live = np.exp(logp) > 0
            H[r] = -(np.exp(logp[live]) * logp[live]).sum()
            lp[r] = 0.0 if tokens[r] == -1 else logp[tokens[r]] if 0 <= tokens[r] < vocab else np.nan
            top[r] = logp[order]
        if not -1 <= tokens[r] < vocab:
            lp[r] = np.nan
    return lp, lse, H, top, ids


def token_logprobs_bwd(logits, tokens, scale, lse, entropy, g, h):
    """Gradient of the logits for given lse and entropy; g, h: gradients of logprob and entropy (None: zero)."""
    rows, vocab = logits.shape
    d = np.zeros((rows, vocab))
    for r in range(rows):
        given = g is not None and 0 <= tokens[r] < vocab
        gr, hr = (float(g[r]) if given else 0.0), (0.0 if h is None else float(h[r]))
        if (gr == 0.0 and hr == 0.0) or np.isneginf(lse[r]):
            continue
        s = np.asarray(logits[r], np.float64) * scale
        logp = s - float(lse[r])
        if abs(lse[r]) >= 8192:  # an fp32 lse of this size has no digits left for p
            logp = s - s.max()
            logp -= np.log(np.exp(logp).sum())
        p = np.exp(logp)
        live = p > 0
        d[r] = -gr * p
        if hr != 0.0:
            d[r][live] -= hr * p[live] * (logp[live] + float(entropy[r]))
        if given:
            d[r, tokens[r]] += gr
        if np.isnan(lse[r]):
            d[r] = np.nan
    return d * scale
