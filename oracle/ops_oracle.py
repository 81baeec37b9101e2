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


# ------------------------------------------------------------------ AdamW
def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step):
    """New p, m, v in fp64."""
    p, g, m, v = (np.asarray(t, np.float64) for t in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * weight_decay * p - lr * update, m, v


def e4m3_values():
    """What the 256 codes stand for: sign, 4 bits of exponent (bias 7, 0 is even spacing of 2^-9), 3 of mantissa;
    exponent and mantissa all ones is NaN."""
    code = np.arange(256)
    exponent, mantissa = (code >> 3) & 15, code & 7
    v = np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent - 10.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code >= 128, -v, v)


def mix32(x):
    x = np.asarray(x, np.uint64) & 0xFFFFFFFF
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def adamw_random_bits(seed, step, place, count):
    """32 bits for every element of the tensor at ``place`` in the list."""
    golden = 0x9E3779B9
    key = mix32(np.uint64((seed + step * golden) & 0xFFFFFFFF))
    key = mix32(key ^ np.uint64(place + 1))
    i = np.arange(count, dtype=np.uint64)
    assert count < 2 ** 32
    return mix32(key + (i * np.uint64(golden) & np.uint64(0xFFFFFFFF)))


def block_scale(x, block=256):
    """Power of two per block that brings the largest finite magnitude into [128, 256), at least 2^-107."""
    out = []
    for b in range(0, len(x), block):
        a = np.abs(x[b:b + block])
        top = a[np.isfinite(a)].max(initial=0.0)
        out.append(2.0 ** (max(np.frexp(top)[1] - 1, -100) - 7) if top > 0 else 2.0 ** -107)
    return np.array(out)


def stochastic_code(y, bits16, keep):
    """e4m3 code below or above y (|y| <= 256), the upper one if the fraction between them, in 2^-20, plus the 16
    random bits (as 2^-20 (16 bits + 1/2)) reaches one; and how far y is from where that changes."""
    values = e4m3_values()[:127]
    a = np.abs(y)
    finite = a <= 256
    a = np.where(finite, a, 0.0)
    low = np.clip(np.searchsorted(values, a, side="right") - 1, 0, 125)
    span = values[low + 1] - values[low]
    fraction = np.floor((a - values[low]) / span * 2 ** 20)
    rest = fraction + bits16 * 16.0 + 8 - 2 ** 20
    code = low + (rest >= 0)
    # the border above, or that of the number's own interval from below
    margin = np.minimum(np.abs(rest), fraction) * span / 2 ** 20
    if keep:
        code = np.where((y > 0) & (code == 0), 1, code)
    return np.where(finite, code + np.where(np.signbit(y), 128, 0), 127).astype(np.uint8), margin


def adamw_states8(g, m_code, v_code, m_scale, v_scale, beta1, beta2, seed, step, place):
    """fp32 m and root that the step uses, the new codes, how far m and root are from where their codes change (fp32
    arithmetic may land on the other side), and the new scales."""
    n = len(g)
    per = lambda s: np.repeat(np.asarray(s, np.float64), 256)[:n]
    value = e4m3_values()
    g = np.asarray(g, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        m = (beta1 * (value[m_code] * per(m_scale)) + (1 - beta1) * g).astype(np.float32)
        v0 = (np.float32(value[v_code] * per(v_scale)) ** 2).astype(np.float64)
        v = (beta2 * v0 + ((1 - beta2) * g) * g).astype(np.float32)
        root = np.sqrt(v)
    bits = adamw_random_bits(seed, step, place, n)
    ms, vs = block_scale(m.astype(np.float64)), block_scale(root.astype(np.float64))

    def scaled(x, s):
        # numbers below 2^-6 get 2^-6 added in fp32 before their fraction is taken, which rounds them to 2^-29
        y = x.astype(np.float64) / per(s)
        small = np.abs(y) < 2.0 ** -6
        with np.errstate(invalid="ignore"):
            z = (np.float32(np.abs(y)) + np.float32(2.0 ** -6)).astype(np.float64) - 2.0 ** -6
        return np.where(small, np.copysign(z, y), y)

    new_m, off_m = stochastic_code(scaled(m, ms), (bits & np.uint64(0xFFFF)).astype(np.float64), False)
    r = scaled(root, vs)
    new_v, off_v = stochastic_code(np.where(root > 0, np.maximum(r, 2.0 ** -30), r) if n else r,
                                   (bits >> np.uint64(16)).astype(np.float64), True)
    return m, root, new_m, new_v, off_m * per(ms), off_v * per(vs), ms, vs
