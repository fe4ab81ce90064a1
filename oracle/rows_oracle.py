"""The operators on rows from their definitions, in 64 bits on the CPU (numpy): test infrastructure only.

Layer norm and its gradients, the row quantiser (whose codes and scales are defined by fp32 steps, repeated here in fp32),
the product of 8-bit integers, log probabilities with entropy and alternatives, and their gradient.  Inputs are float64
arrays that hold the stored values exactly.
"""
import numpy as np

INV127 = np.float32(1.0) / np.float32(127.0)
LEAST_SCALE = np.float32(2.0 ** -126)


def layernorm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def layernorm_bwd(x, dy, gamma, mean, rstd):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (g - g.mean(1)[:, None] - xh * (g * xh).mean(1)[:, None])
    return dx, (dy * xh).sum(0), dy.sum(0)


def quantize_rows(x32):
    """fp32 rows -> (codes, scales): the definition's own fp32 steps."""
    x32 = np.asarray(x32, dtype=np.float32)
    with np.errstate(all="ignore"):
        amax = np.abs(x32).max(1)
        scale = np.maximum(amax * INV127, LEAST_SCALE).astype(np.float32)
        inv = (np.float32(1.0) / scale).astype(np.float32)
        good = np.isfinite(x32).all(1)
        codes = np.rint(np.where(good[:, None], x32 * inv[:, None], np.float32(0.0)))
    return codes.astype(np.int8), np.where(good, scale, np.float32(np.nan)).astype(np.float32)


def int_linear(a, a_scale, w, w_scale, bias, relu):
    """int8 codes, fp32 scales and bias -> float64 result, and the size of what is rounded on the way."""
    acc = (a.astype(np.int64) @ w.astype(np.int64).T).astype(np.float64)
    v = acc * (a_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)[None, :])
    size = np.abs(v)
    if bias is not None:
        v = v + bias.astype(np.float64)
        size = size + np.abs(bias.astype(np.float64))
    return (np.where(v < 0, 0.0, v) if relu else v), size


def order_key(x):
    """Sort keys, the likeliest first: by value (NaN above all), the lower index first among equals."""
    return np.where(np.isnan(x), -np.inf, -x), ~np.isnan(x)


def logprob(x, target, top):
    """-> dict of logp, lse, entropy, top_id, top_logp."""
    rows, cols = x.shape
    out = {"logp": np.zeros(rows), "lse": np.zeros(rows), "entropy": np.zeros(rows),
           "top_id": np.zeros((rows, top), dtype=np.int64), "top_logp": np.zeros((rows, top))}
    for t in range(rows):
        v = x[t]
        neg, nan_last = order_key(v)
        ids = np.lexsort((np.arange(cols), nan_last, neg))[:top]
        if np.isnan(v).any() or np.isposinf(v).any():
            lse = h = np.nan
        elif np.isneginf(v).all():
            lse, h = -np.inf, 0.0
        else:
            m = v.max()
            e = np.exp(v - m)
            lse = m + np.log(e.sum())
            p = e / e.sum()
            h = float(np.sum(np.where(p > 0, p * (lse - np.where(p > 0, v, 0.0)), 0.0)))
        out["lse"][t], out["entropy"][t], out["top_id"][t] = lse, h, ids
        empty = np.isneginf(lse)
        out["top_logp"][t] = -np.inf if empty else v[ids] - lse
        k = int(target[t]) if target is not None else -1
        out["logp"][t] = 0.0 if k < 0 else np.nan if k >= cols else -np.inf if empty else v[k] - lse
    return out


def logprob_bwd(x, target, lse, entropy, g_logp, g_entropy):
    rows, cols = x.shape
    dx = np.zeros_like(x)
    for t in range(rows):
        if np.isneginf(lse[t]):
            continue
        k = int(target[t]) if g_logp is not None else -1
        g = 0.0 if k < 0 else np.nan if k >= cols else g_logp[t]
        lp = x[t] - lse[t]
        p = np.exp(lp)
        hit = (np.arange(cols) == k).astype(np.float64)
        dx[t] = g * (hit - p)
        if g_entropy is not None:
            dx[t] -= g_entropy[t] * np.where(p > 0, p * (np.where(p > 0, lp, 0.0) + entropy[t]), 0.0)
    return dx
