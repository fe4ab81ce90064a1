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


def activation(z, act):
    """-> (act(z), its slope); the slope of ReLU at 0 is 0."""
    from scipy.special import erfc

    if act == "relu":
        return np.where(z < 0, 0.0, z), np.where(z > 0, 1.0, np.where(z <= 0, 0.0, z))
    if act == "gelu":
        phi = 0.5 * erfc(-z * np.sqrt(0.5))
        return z * phi, phi + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    if act == "silu":
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    return z, np.ones_like(z)


def linear(x, w, bias, residual, act):
    """-> (out, pre, size): size is the sum of the magnitudes that pre adds up."""
    z, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        z, size = z + bias, size + np.abs(bias)
    out = activation(z, act)[0]
    return (out if residual is None else out + residual), z, size


def linear_bwd(x, w, pre, dout, act):
    """-> (dx, dw, dbias)."""
    dz = dout if act == "none" else dout * activation(pre, act)[1]
    return dz @ w, dz.T @ x, dz.sum(0)


def row_norm(x, rms, eps):
    """-> (normed rows, mean, rstd)."""
    mean = np.zeros(len(x)) if rms else x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None], mean, rstd


def residual_norm(r, h, gate, gate_rows, sigmoid, gamma_h, beta_h, scale, gamma, beta, post, rms, eps):
    """-> (sum, y, stats, branch): branch is what was added to r.  gamma_h .. beta are arrays, or None for ones or zeros."""
    one = lambda v: 1.0 if v is None else v  # noqa: E731
    zero = lambda v: 0.0 if v is None else v  # noqa: E731
    u, mean_h, rstd_h = row_norm(h, rms, eps) if post else (h, np.zeros(len(h)), np.ones(len(h)))
    if post:
        u = u * one(gamma_h) + zero(beta_h)
    if gate is not None:
        g = gate[np.arange(len(h)) // gate_rows]
        u = u * (1.0 / (1.0 + np.exp(-g)) if sigmoid else g)
    branch = u * one(scale)
    xh, mean, rstd = row_norm(r + branch, rms, eps)
    return r + branch, xh * one(gamma) + zero(beta), np.stack([mean_h, rstd_h, mean, rstd], 1), branch


def residual_norm_bwd(x, h, gate, gate_rows, sigmoid, gamma_h, beta_h, scale, gamma, stats, dr_out, dy, post, rms):
    """-> dict of dr, dh, dgate, dgamma_h, dbeta_h, dscale, dgamma, dbeta."""
    one = lambda v: 1.0 if v is None else v  # noqa: E731
    zero = lambda v: 0.0 if v is None else v  # noqa: E731

    def through(g, xh, rstd):
        return rstd[:, None] * (g - (0.0 if rms else g.mean(1)[:, None]) - xh * (g * xh).mean(1)[:, None])

    out = {}
    xh = (x - stats[:, 2:3]) * stats[:, 3:4]
    out["dr"] = dr = dr_out + through(dy * one(gamma), xh, stats[:, 3])
    out["dgamma"], out["dbeta"] = (dy * xh).sum(0), dy.sum(0)
    hh = (h - stats[:, 0:1]) * stats[:, 1:2] if post else h
    u = hh * one(gamma_h) + zero(beta_h) if post else h
    p = dr
    if gate is not None:
        at = np.arange(len(h)) // gate_rows
        s = 1.0 / (1.0 + np.exp(-gate)) if sigmoid else gate
        d = np.zeros_like(gate)
        np.add.at(d, at, dr * u * one(scale))
        out["dgate"] = d * s * (1.0 - s) if sigmoid else d
        p = dr * s[at]
    du = p * one(scale)
    out["dscale"] = (p * u).sum(0)
    out["dgamma_h"], out["dbeta_h"] = (du * hh).sum(0), du.sum(0)
    out["dh"] = through(du * one(gamma_h), hh, stats[:, 1]) if post else du
    return out


def newton_schulz(x, steps, coefficients, eps):
    """One matrix."""
    a, b, c = coefficients
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        m = x @ x.T
        x = a * x + (b * m + c * (m @ m)) @ x
    return x
