"""Oracle of the calls around attention and verification: NumPy, fp64, from the definitions in include/tslt.h; it shares no code with csrc/."""
from __future__ import annotations

import numpy as np


# ---- norms and rotation -----------------------------------------------------------------------------------------

def turns(position, freq):
    """cos and sin of position * freq, [..., pairs]: the product and the functions in extended precision."""
    angle = np.asarray(position, dtype=np.longdouble) * np.asarray(freq, dtype=np.longdouble)
    return np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)


def pair_channels(rotary, adjacent):
    j = np.arange(rotary // 2)
    return (2 * j, 2 * j + 1) if adjacent else (j, j + rotary // 2)


def token_positions(B, n, pairs, position, base, axis):
    """[B, n, pairs] whole numbers."""
    at = np.broadcast_to(np.arange(n, dtype=np.int64)[None, :, None], (B, n, 1)) if position is None else np.broadcast_to(position.astype(np.int64), (B, n, position.shape[2]))
    if base is not None:
        at = at + base.astype(np.int64)[:, None, None]
    named = np.zeros(pairs, dtype=np.int64) if axis is None else np.clip(axis.astype(np.int64), 0, at.shape[2] - 1)
    return at[:, :, named] if at.shape[2] > 1 else np.broadcast_to(at, (B, n, pairs))


def rotate(x, cos, sin, adjacent, weight=None, eps=None):
    """x [B, n, heads, D]; cos, sin [B, n, pairs].  eps None: no norm."""
    x = np.asarray(x, dtype=np.float64)
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight
    y = x.copy()
    u, v = pair_channels(2 * cos.shape[-1], adjacent)
    c, s = cos[:, :, None], sin[:, :, None]
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    return y


def rotate_backward(g, x, cos, sin, adjacent, weight=None, eps=None):
    """Gradients of x and of the weight (None without a norm)."""
    g = rotate(g, cos, -sin, adjacent)
    if eps is None:
        return g, None
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dw = (g * x * r).sum((0, 1, 2))
    h = g if weight is None else g * weight
    return r * h - x * r ** 3 * (h * x).mean(-1, keepdims=True), dw


# ---- log probabilities ------------------------------------------------------------------------------------------

def inverse_temperature(T):
    return float(np.float32(1.0) / np.float32(T))


def logprob_row(z, rT, token, top):
    """One row: dict of logp, entropy, lse, top_idx, top_logp, status (1: not finite, 2: empty)."""
    z = np.asarray(z, dtype=np.float64)
    none = dict(logp=np.nan, entropy=np.nan, lse=np.nan, top_idx=np.full(top, -1), top_logp=np.full(top, -np.inf))
    if np.isnan(z).any() or np.isposinf(z).any():
        return dict(none, status=1)
    if np.isneginf(z).all():
        return dict(none, lse=-np.inf, status=2)
    m = z.max()
    d = (z - m) * rT                                   # (of numbers near fp32's largest, lse itself has no room for ln S)
    ln_S = np.log(np.exp(d).sum())
    lse = m * rT + ln_S
    logp = d - ln_S
    p = np.exp(logp)
    seen = p > 0
    order = np.lexsort((np.arange(z.size), -z))[:top]
    order = order[z[order] > -np.inf]
    idx, val = np.full(top, -1), np.full(top, -np.inf)
    idx[:order.size], val[:order.size] = order, logp[order]
    return dict(logp=logp[token] if 0 <= token < z.size else np.nan, entropy=-(p[seen] * logp[seen]).sum(), lse=lse, top_idx=idx, top_logp=val, status=0)


def logprob_backward_row(z, rT, token, lse, entropy, top_idx, g_logp, g_entropy, g_lse, g_top):
    """The gradient of one row of logits; None stands for a gradient that is not there."""
    z = np.asarray(z, dtype=np.float64)
    if not np.isfinite(lse):
        return np.full(z.size, np.nan)
    d = z * rT - lse
    p = np.exp(d)
    out = np.zeros(z.size)
    if g_logp is not None and 0 <= token < z.size:
        out -= g_logp * p
        out[token] += g_logp
    if g_entropy is not None:
        out -= g_entropy * p * np.where(p > 0, d + entropy, 0.0)
    if g_lse is not None:
        out += g_lse * p
    if g_top is not None:
        for i, g in zip(top_idx, g_top):
            if 0 <= i < z.size:
                out -= g * p
                out[i] += g
    return out * rT


# ---- adapters ---------------------------------------------------------------------------------------------------

def adapt(x, base, a, b, adapter, scale=None, rank=None):
    """x [B, n, K], base [B, n, N], a [adapters, R, K], b [adapters, N, R]."""
    out = np.array(base, dtype=np.float64)
    for s, i in enumerate(adapter):
        if 0 <= i < a.shape[0]:
            r = a.shape[1] if rank is None else min(max(int(rank[i]), 0), a.shape[1])
            f = 1.0 if scale is None else float(scale[i])
            out[s] += f * ((np.asarray(x[s], dtype=np.float64) @ np.asarray(a[i, :r], dtype=np.float64).T) @ np.asarray(b[i, :, :r], dtype=np.float64).T)
    return out
